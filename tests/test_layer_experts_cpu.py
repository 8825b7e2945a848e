"""Norm, sorted experts, their products and the clipped gradient without a GPU: structures, refusals, the differentiable forms over
stand-ins for the kernels, and the clipping of sharded gradients over two gloo ranks.

A refusal is returned before anything touches a device, so the addresses in these calls are never used."""
import ctypes as C
import math
import os
import struct

import pytest
import torch

from paper_2407_04480_b200 import build as loco_build
from paper_2407_04480_b200 import exchange, layer, loco
from tests.test_multirank_cpu import _free_port

PTR = 1 << 20                    # 16-byte aligned, never read


@pytest.fixture(scope="module", autouse=True)
def built():
    loco_build.build()


def test_packed_structures_have_the_sizes_of_the_c_ones():
    def fields(*names):
        return type("S", (C.Structure,), {"_fields_": list(names)})
    rows = fields(("ptr", C.c_void_p), ("s", C.c_int64))
    norm = fields(*((n, C.c_int32) for n in ("dtype", "dim", "bits8", "block")), ("eps", C.c_float))
    experts = fields(*((n, C.c_int32) for n in ("dtype", "dim", "k")), ("tokens", C.c_int64), ("rows", C.c_int64))
    matrices = fields(("ptr", C.c_void_p), ("e", C.c_int64), ("r", C.c_int64))
    product = fields(("experts", C.c_int32), ("rows", C.c_int64), ("d_in", C.c_int32), ("d_out", C.c_int32), ("t", C.c_int32))
    span = fields(("x", C.c_void_p), ("y", C.c_void_p), ("n", C.c_uint64), ("dtype", C.c_int32))
    for packed, made in ((layer._ROWS, rows), (layer._NORM, norm), (layer._EXPERTS, experts), (layer._MATRICES, matrices), (layer._PRODUCT, product),
                         (layer._SPAN, span)):
        assert packed.size == C.sizeof(made)
    p = product.from_buffer_copy(layer._PRODUCT.pack(1, 2, 3, 4, 5))
    assert [getattr(p, n) for n, _ in product._fields_] == [1, 2, 3, 4, 5]
    e = experts.from_buffer_copy(layer._EXPERTS.pack(1, 2, 3, 4, 5))
    assert [getattr(e, n) for n, _ in experts._fields_] == [1, 2, 3, 4, 5]
    s = span.from_buffer_copy(layer._SPAN.pack(1, 2, 3, 4))
    assert [getattr(s, n) for n, _ in span._fields_] == [1, 2, 3, 4]


def rows(ptr=PTR, stride=64):
    return struct.pack("@Pq", ptr, stride)


# ---- norm ------------------------------------------------------------------------------------

def norm_cfg(dtype=loco.BF16, dim=64, bits8=0, block=0, eps=1e-5):
    return layer._NORM.pack(dtype, dim, bits8, block, eps)


def forward(cfg, n=4, x=rows(), r=None, w=None, total=None, y=rows(), scale=None):
    return layer.lib().loco_norm_forward(cfg, n, x, r, w, total, y, scale, None)


def backward(cfg, n=4, h=rows(), dy=rows(), w=None, dt=None, dx=rows(), dw=None, work=None, size=0):
    return layer.lib().loco_norm_backward(cfg, n, h, dy, w, dt, dx, dw, work, size, None)


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=2), loco.ERR_ARG), (dict(dim=0), loco.ERR_ARG), (dict(dim=16385), loco.ERR_UNSUPPORTED), (dict(eps=-1.0), loco.ERR_ARG),
    (dict(eps=math.nan), loco.ERR_ARG), (dict(eps=math.inf), loco.ERR_ARG), (dict(bits8=1, block=64), loco.ERR_ARG), (dict(bits8=1, block=-1), loco.ERR_ARG)])
def test_norm_refuses_a_bad_configuration(bad, code):
    assert forward(norm_cfg(**bad), scale=PTR) == code
    assert layer.lib().loco_norm_backward_workspace_bytes(norm_cfg(**bad)) == 0


def test_norm_refuses_bad_operands():
    ok = norm_cfg()
    assert forward(None) == loco.ERR_ARG and forward(ok, n=-1) == loco.ERR_ARG
    assert forward(ok, x=None) == loco.ERR_ARG and forward(ok, y=rows(ptr=0)) == loco.ERR_ARG
    assert forward(ok, r=rows()) == loco.ERR_ARG and forward(ok, total=rows()) == loco.ERR_ARG
    assert forward(ok, y=rows(stride=63)) == loco.ERR_ARG and forward(ok, y=rows(stride=0)) == loco.ERR_ARG and forward(ok, x=rows(stride=-64)) == loco.ERR_ARG
    assert forward(ok, r=rows(), total=rows(stride=0)) == loco.ERR_ARG
    assert forward(ok, x=rows(ptr=PTR + 1)) == loco.ERR_ALIGN and forward(ok, w=PTR + 1) == loco.ERR_ALIGN
    assert forward(norm_cfg(bits8=1)) == loco.ERR_ARG and forward(norm_cfg(bits8=1, block=128), scale=PTR + 2) == loco.ERR_ALIGN
    assert forward(ok, n=0, x=rows(ptr=0), y=rows(ptr=0)) == loco.OK
    need = layer.lib().loco_norm_backward_workspace_bytes(ok)
    assert need >= 64 * 4
    assert backward(None) == loco.ERR_ARG and backward(ok, n=-1) == loco.ERR_ARG and backward(norm_cfg(bits8=1)) == loco.ERR_ARG
    for name in ("h", "dy", "dx"):
        assert backward(ok, **{name: None}) == loco.ERR_ARG and backward(ok, **{name: rows(ptr=PTR + 1)}) == loco.ERR_ALIGN
    assert backward(ok, dx=rows(stride=0)) == loco.ERR_ARG and backward(ok, dt=rows(ptr=0)) == loco.ERR_ARG
    assert backward(ok, dw=PTR) == loco.ERR_ARG and backward(ok, dw=PTR, work=PTR, size=need - 1) == loco.ERR_SIZE
    assert backward(ok, dw=PTR, work=PTR + 8, size=need) == loco.ERR_ALIGN and backward(ok, dw=PTR + 1, work=PTR, size=need) == loco.ERR_ALIGN
    assert backward(ok, n=0) == loco.OK


# ---- experts ---------------------------------------------------------------------------------

def test_sort_refuses_bad_arguments():
    need = layer.lib().loco_experts_sort_workspace_bytes(8)
    call = lambda e=8, t=4, k=2, i=PTR, o=PTR, p=PTR, w=PTR, n=need: layer.lib().loco_experts_sort(e, t, k, i, o, p, w, n, None)
    for bad in (dict(e=0), dict(e=513), dict(t=-1), dict(k=0), dict(k=17), dict(t=1 << 30, k=2), dict(i=None), dict(o=None), dict(p=None), dict(w=None)):
        assert call(**bad) == loco.ERR_ARG, bad
    for bad in (dict(i=PTR + 2), dict(o=PTR + 1), dict(p=PTR + 2), dict(w=PTR + 8)):
        assert call(**bad) == loco.ERR_ALIGN, bad
    assert call(n=need - 1) == loco.ERR_SIZE
    assert layer.lib().loco_experts_sort_workspace_bytes(0) == 0 and layer.lib().loco_experts_sort_workspace_bytes(513) == 0


def test_moves_refuse_bad_arguments():
    L = layer.lib()

    def cfg(dtype=loco.BF16, dim=64, k=2, tokens=4, n=8):
        return layer._EXPERTS.pack(dtype, dim, k, tokens, n)
    calls = {"dispatch": lambda c, a=rows(), p=PTR, b=rows(), w=PTR: L.loco_experts_dispatch(c, a, p, b, None),
             "combine": lambda c, a=rows(), p=PTR, b=rows(), w=PTR: L.loco_experts_combine(c, b, p, w, a, None),
             "backward": lambda c, a=rows(), p=PTR, b=rows(), w=PTR: L.loco_experts_combine_backward(c, a, rows(), p, w, b, PTR, None)}
    for name, call in calls.items():
        for bad in (dict(dtype=3), dict(dim=0), dict(k=0), dict(k=17), dict(tokens=-1), dict(tokens=1 << 30), dict(n=-1), dict(n=1 << 31)):
            assert call(cfg(**bad)) == loco.ERR_ARG, (name, bad)
        assert call(cfg(dim=(1 << 30) + 8), a=rows(stride=1 << 31), b=rows(stride=1 << 31)) == loco.ERR_UNSUPPORTED
        assert call(None) == loco.ERR_ARG and call(cfg(), p=None) == loco.ERR_ARG and call(cfg(), a=None) == loco.ERR_ARG and call(cfg(), b=rows(ptr=0)) == loco.ERR_ARG
        assert call(cfg(), p=PTR + 2) == loco.ERR_ALIGN and call(cfg(), a=rows(ptr=PTR + 1)) == loco.ERR_ALIGN and call(cfg(), b=rows(ptr=PTR + 1)) == loco.ERR_ALIGN
        assert call(cfg(tokens=0), a=rows(ptr=0), p=None) == loco.OK
    assert calls["dispatch"](cfg(), b=rows(stride=32)) == loco.ERR_ARG and calls["combine"](cfg(), a=rows(stride=0)) == loco.ERR_ARG
    assert calls["combine"](cfg(), w=PTR + 2) == loco.ERR_ALIGN and calls["backward"](cfg(), w=None) == loco.ERR_ARG
    clear = lambda dtype=loco.BF16, d=64, n=4, r=rows(), e=8, o=PTR: L.loco_experts_clear(dtype, d, n, r, e, o, None)
    for bad in (dict(dtype=2), dict(d=0), dict(n=-1), dict(r=None), dict(r=rows(stride=0)), dict(e=0), dict(o=None)):
        assert clear(**bad) == loco.ERR_ARG, bad
    assert clear(o=PTR + 2) == loco.ERR_ALIGN and clear(r=rows(ptr=PTR + 1)) == loco.ERR_ALIGN and clear(n=0, r=rows(ptr=0)) == loco.OK


def matrices(ptr=PTR, e=64 * 64, r=64):
    return struct.pack("@Pqq", ptr, e, r)


def test_product_refuses_bad_arguments():
    L = layer.lib()

    def cfg(experts=4, n=100, d_in=64, d_out=64, t=0):
        return layer._PRODUCT.pack(experts, n, d_in, d_out, t)
    plain = lambda c, a=rows(), w=matrices(), o=PTR, y=rows(): L.loco_experts_product(c, a, w, o, y, None)
    weights = lambda c, a=rows(), w=matrices(), o=PTR, y=rows(): L.loco_experts_product_weights(c, a, y, o, w, None)
    for call in (plain, weights):
        for bad in (dict(experts=0), dict(experts=513), dict(n=-1), dict(n=1 << 31), dict(d_in=0), dict(d_out=-8)):
            assert call(cfg(**bad)) == loco.ERR_ARG, bad
        assert call(cfg(d_in=(1 << 30) + 8)) == loco.ERR_UNSUPPORTED and call(cfg(d_out=(1 << 30) + 8)) == loco.ERR_UNSUPPORTED
        assert call(cfg(d_in=60)) == loco.ERR_UNSUPPORTED and call(cfg(d_out=4)) == loco.ERR_UNSUPPORTED
        assert call(None) == loco.ERR_ARG and call(cfg(), o=None) == loco.ERR_ARG and call(cfg(), a=None) == loco.ERR_ARG and call(cfg(), w=None) == loco.ERR_ARG
        for bad in (dict(a=rows(ptr=PTR + 8)), dict(a=rows(stride=68)), dict(y=rows(ptr=PTR + 2)), dict(w=matrices(ptr=PTR + 8)), dict(w=matrices(r=68)),
                    dict(w=matrices(e=64 * 64 + 4)), dict(o=PTR + 2)):
            assert call(cfg(), **bad) == loco.ERR_ALIGN, bad
        for bad in (dict(a=rows(stride=-64)), dict(w=matrices(r=-64)), dict(w=matrices(e=-8)), dict(w=matrices(ptr=0)), dict(a=rows(stride=1 << 39))):
            assert call(cfg(), **bad) == loco.ERR_ARG, bad
    assert plain(cfg(), y=rows(stride=0)) == loco.ERR_ARG and weights(cfg(), w=matrices(e=0)) == loco.ERR_ARG and weights(cfg(), w=matrices(r=32)) == loco.ERR_ARG
    assert plain(cfg(n=0), a=rows(ptr=0), y=rows(ptr=0)) == loco.OK


def test_gradient_refuses_bad_lists():
    L = layer.lib()
    span = lambda x=PTR, y=PTR, n=8, dtype=loco.BF16: layer._SPAN.pack(x, y, n, dtype)
    need = L.loco_gradient_squares_workspace_bytes()
    squares = lambda s=span(), k=1, q=PTR, w=PTR, n=need: L.loco_gradient_squares(s, k, q, w, n, None)
    clip = lambda s=span(), k=1, q=PTR, m=1.0, norm=PTR: L.loco_gradient_clip(s, k, q, m, norm, None)
    for call in (squares, clip):
        for bad in (dict(k=-1), dict(s=None), dict(q=None), dict(s=span(dtype=2)), dict(s=span(x=0)), dict(s=span(n=1 << 50))):
            assert call(**bad) == loco.ERR_ARG, bad
        assert call(s=span(x=PTR + 1)) == loco.ERR_ALIGN and call(q=PTR + 4) == loco.ERR_ALIGN
        assert call(s=span() + span(dtype=5), k=2) == loco.ERR_ARG                # the last of a list
    assert squares(w=None) == loco.ERR_ARG and squares(w=PTR + 8) == loco.ERR_ALIGN and squares(n=need - 1) == loco.ERR_SIZE
    assert clip(s=span(y=0)) == loco.ERR_ARG and clip(s=span(y=PTR + 1)) == loco.ERR_ALIGN and clip(norm=PTR + 2) == loco.ERR_ALIGN
    assert clip(m=-1.0) == loco.ERR_ARG and clip(m=math.nan) == loco.ERR_ARG


def test_an_empty_list_of_gradients_is_refused():
    with pytest.raises(ValueError):
        layer.clip_gradients([], 1.0)
    with pytest.raises(ValueError):
        exchange.clip_shards([], 1.0)


# ---- differentiable forms over stand-ins -----------------------------------------------------

def plain_norm(x, w, eps):
    y = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + eps)
    return y if w is None else y * w


@pytest.fixture
def kernels(monkeypatch):
    """The calls' formulas in plain torch, in the type of the operands."""
    calls = []

    def stand_in(name):
        def place(fn):
            monkeypatch.setattr(layer, name, lambda *a, **k: (calls.append(name), fn(*a, **k))[1])
        return place

    @stand_in("loco_norm_forward")
    def _(x, y, weight=None, residual=None, total=None, eps=1e-5):
        h = x if residual is None else x + residual
        if total is not None:
            total.copy_(h)
        y.copy_(plain_norm(h, weight, eps))

    @stand_in("loco_norm_backward")
    def _(h, dy, dx, work=None, weight=None, dweight=None, dtotal=None, eps=1e-5):
        r = torch.rsqrt(h.square().mean(1, keepdim=True) + eps)
        n, g = h * r, dy if weight is None else dy * weight
        dx.copy_(r * (g - n * (g * n).mean(1, keepdim=True)) + (0 if dtotal is None else dtotal))
        if dweight is not None:
            dweight.copy_((dy * n).sum(0))

    @stand_in("loco_experts_clear")
    def _(rows, offsets):
        rows[int(offsets[-1]):] = 0

    @stand_in("loco_experts_dispatch")
    def _(x, place, rows):
        rows.fill_(math.nan)                         # what nothing has been written to
        for t, p in enumerate(place.tolist()):
            for r in p:
                if r >= 0:
                    rows[r] = x[t]

    @stand_in("loco_experts_combine")
    def _(rows, place, y, weight=None):
        for t, p in enumerate(place.tolist()):
            y[t] = sum(((1.0 if weight is None else weight[t, j]) * rows[r] for j, r in enumerate(p) if r >= 0), torch.zeros_like(y[t]))

    @stand_in("loco_experts_combine_backward")
    def _(dy, rows, place, weight, drows, dweight):
        drows.fill_(math.nan)
        dweight.zero_()
        for t, p in enumerate(place.tolist()):
            for j, r in enumerate(p):
                if r >= 0:
                    drows[r], dweight[t, j] = weight[t, j] * dy[t], (dy[t] * rows[r]).sum()

    @stand_in("loco_experts_product")
    def _(x, w, offsets, y, transposed=False):
        y.fill_(math.nan)
        for e in range(len(w)):
            at = slice(int(offsets[e]), int(offsets[e + 1]))
            y[at] = x[at] @ (w[e].T if transposed else w[e])

    @stand_in("loco_experts_product_weights")
    def _(a, b, offsets, dw):
        for e in range(len(dw)):
            at = slice(int(offsets[e]), int(offsets[e + 1]))
            dw[e] = a[at].T @ b[at]
    return calls


def normal(*shape, seed=0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


@pytest.mark.parametrize("weight", [True, False])
@pytest.mark.parametrize("used", ["both", "norm", "total"])
def test_norm_form_has_the_gradient_of_the_formula(kernels, weight, used):
    x, r, w = normal(2, 3, 8).requires_grad_(), normal(2, 3, 8, seed=1).requires_grad_(), normal(8, seed=2).requires_grad_()
    leaves = [x, r] + ([w] if weight else [])
    gy, gt = normal(2, 3, 8, seed=3), normal(2, 3, 8, seed=4)

    def loss(y, total):
        return sum(t.mul(g).sum() for t, g, name in ((y, gy, "norm"), (total, gt, "total")) if used in ("both", name))
    got = torch.autograd.grad(loss(*layer.norm(x, w if weight else None, residual=r)), leaves, allow_unused=True)
    want = torch.autograd.grad(loss(plain_norm(x + r, w if weight else None, 1e-5), x + r), leaves, allow_unused=True)
    for a, b in zip(got, want):
        assert torch.allclose(torch.zeros(()).double() if a is None else a, torch.zeros(()).double() if b is None else b)
    y = layer.norm(x)                                # without a residual: one result
    got, = torch.autograd.grad(y, x, gy)
    want, = torch.autograd.grad(plain_norm(x, None, 1e-5), x, gy)
    assert torch.allclose(got, want)


@pytest.mark.parametrize("weighted", [True, False])
@pytest.mark.parametrize("transposed", [True, False])
def test_expert_forms_have_the_gradient_of_the_formulas(kernels, weighted, transposed):
    """Three experts, one of them idle, a token without choices, a choice left out; the same with a product per choice."""
    index = torch.tensor([[0, 2], [2, 0], [-1, -1], [2, -1]])
    place = torch.tensor([[0, 2], [3, 1], [-1, -1], [4, -1]], dtype=torch.int32)
    offsets = torch.tensor([0, 2, 2, 5], dtype=torch.int32)
    x, weight = normal(4, 8).requires_grad_(), normal(4, 2, seed=1).requires_grad_()
    w = normal(3, 16, 8, seed=2) if transposed else normal(3, 8, 16, seed=2)
    w.requires_grad_()
    rows = layer.dispatch(x, place, offsets)
    assert rows.shape == (8, 8) and not rows[5:].any()
    mid = layer.experts_product(rows, w, offsets, transposed=transposed)
    assert torch.isfinite(mid).all() and not mid[5:].any()
    y = layer.combine(mid.tanh(), place, offsets, weight if weighted else None)
    plain = torch.stack([sum((((weight[t, j] if weighted else 1.0) * (x[t] @ (w[e].T if transposed else w[e])).tanh()) for j, e in enumerate(index[t].tolist()) if e >= 0),
                             torch.zeros(16, dtype=torch.float64)) for t in range(4)])
    assert torch.allclose(y, plain)
    g, leaves = normal(4, 16, seed=3), [x, w] + ([weight] if weighted else [])
    for a, b in zip(torch.autograd.grad(y, leaves, g), torch.autograd.grad(plain, leaves, g)):
        assert torch.allclose(a.double(), b, rtol=1e-6)              # the weights' gradient is fp32


def test_product_form_computes_only_what_is_wanted(kernels):
    offsets = torch.tensor([0, 2], dtype=torch.int32)
    for wanted, call in ((0, "loco_experts_product"), (1, "loco_experts_product_weights")):
        x, w = normal(2, 8), normal(1, 8, 8)
        leaf = (x, w)[wanted].requires_grad_()
        y = layer.experts_product(x, w, offsets)
        del kernels[:]
        torch.autograd.grad(y, leaf, torch.ones_like(y))
        assert [k for k in kernels if k.startswith("loco_experts_product")] == [call]


def test_a_second_derivative_is_refused(kernels):
    place, offsets = torch.tensor([[0], [1]], dtype=torch.int32), torch.tensor([0, 2], dtype=torch.int32)
    x, w, weight = normal(2, 8).requires_grad_(), normal(1, 8, 8), normal(2, 1, seed=1)
    for form in (lambda: layer.norm(x), lambda: layer.norm(x, residual=x.detach())[0], lambda: layer.dispatch(x, place, offsets),
                 lambda: layer.combine(x, place, offsets, weight), lambda: layer.experts_product(x, w, offsets)):
        grad, = torch.autograd.grad((form() ** 3).sum(), x, create_graph=True)
        with pytest.raises(RuntimeError, match="differentiated once"):
            torch.autograd.grad((grad ** 2).sum(), x)


def test_forms_notice_places_and_offsets_that_change_before_the_backward_pass(kernels):
    place, offsets = torch.tensor([[0], [1]], dtype=torch.int32), torch.tensor([0, 2], dtype=torch.int32)
    x, w = normal(2, 8).requires_grad_(), normal(1, 8, 8)
    for form, changed in ((lambda: layer.dispatch(x, place, offsets), place), (lambda: layer.combine(x, place, offsets, normal(2, 1)), place),
                          (lambda: layer.experts_product(x, w, offsets), offsets)):
        y = form()
        changed += 0
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.sum().backward()


def test_product_form_takes_a_gradient_that_is_a_view_off_every_boundary(kernels, monkeypatch):
    seen, call = [], layer.loco_experts_product
    monkeypatch.setattr(layer, "loco_experts_product", lambda x, *a, **k: (seen.append(x), call(x, *a, **k)))
    x, w = normal(2, 8).requires_grad_(), normal(1, 8, 8)
    y = layer.experts_product(x, w, torch.tensor([0, 2], dtype=torch.int32))
    joined = torch.cat([torch.zeros(1, dtype=torch.float64), y.flatten()])
    torch.autograd.grad(joined, x, normal(17, seed=3))
    assert seen[-1].is_contiguous() and seen[-1].data_ptr() % 16 == 0


# ---- sharded gradients -----------------------------------------------------------------------

def _squares(gradients, squares, work):
    squares.fill_(sum(float(g.double().square().sum()) for g in gradients))


def _clip(gradients, outputs, squares, norm, max_norm):
    n = math.sqrt(float(squares))
    norm.fill_(n)
    for x, y in zip(gradients, outputs):
        y.copy_(x * (max_norm / n if n > max_norm else 1.0))


def _rank(rank, world, port, out):
    import torch.distributed as dist
    os.environ.update(MASTER_ADDR="127.0.0.1", MASTER_PORT=str(port))
    dist.init_process_group("gloo", rank=rank, world_size=world)
    try:
        layer.loco_gradient_squares, layer.loco_gradient_clip = _squares, _clip
        g = torch.Generator().manual_seed(9)
        whole = torch.randn(1001, generator=g)
        shards = [whole[:500][rank::world].clone(), whole[500:][rank::world].clone()]
        norm = exchange.clip_shards(shards, 2.0, work=torch.zeros(1))
        torch.save((norm, shards), os.path.join(out, "%d.pt" % rank))
    finally:
        dist.destroy_process_group()


def test_shards_are_clipped_to_the_norm_of_the_whole_gradient(tmp_path):
    torch.multiprocessing.spawn(_rank, args=(2, _free_port(), str(tmp_path)), nprocs=2)
    whole = torch.randn(1001, generator=torch.Generator().manual_seed(9))
    got = [torch.load(tmp_path / ("%d.pt" % r)) for r in range(2)]
    n = float(whole.double().norm())
    for r, (norm, shards) in enumerate(got):
        assert abs(float(norm) - n) <= 2e-7 * n
        for part, shard in zip((whole[:500], whole[500:]), shards):
            assert torch.allclose(shard, part[r::2] * (2.0 / n), rtol=1e-6)
    assert abs(math.sqrt(sum(float(s.double().square().sum()) for _, shards in got for s in shards)) - 2.0) < 1e-5
