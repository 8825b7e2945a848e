"""The decoder-layer operators on the GPU where they meet other work: launches in a row, values that are not finite, refusals."""
import ctypes
import math
import os
import subprocess

import pytest
import torch

from paper_2407_04480_b200 import build as loco_build
from paper_2407_04480_b200 import layer, loco
from tests import layer_reference as ref

pytestmark = pytest.mark.gpu

U = ref.U                        # of a rounding to bfloat16, relative
BF, F32 = torch.bfloat16, torch.float32


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(g, *shape, dtype=BF):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("h,hk,d", [(4, 2, 128), (6, 6, 64)])
def test_attention_calls_in_a_row_read_what_the_launch_before_wrote(h, hk, d, packed):
    """Operands, lengths and statistics come from the launches right before; every result has to be what calls with pauses give."""
    g, n = gen(41), [310, 0, 7, 128, 259, 1]
    lead = (sum(n),) if packed else (len(n), max(n))
    src = [normal(g, *lead, x, d) for x in (h, hk, hk, h)]
    lens = torch.tensor(n, device="cuda", dtype=torch.int32)
    cu = torch.tensor([0] + n, device="cuda").cumsum(0).to(torch.int32)

    def chain(pause):
        if packed:
            at = torch.zeros_like(cu)
            at.copy_(cu)
            kw = dict(cu_q=at, cu_k=at, max_q=max(n), max_k=max(n))
        else:
            at = torch.zeros_like(lens)
            at.copy_(lens)
            kw = dict(len_q=at, len_k=at)
        pause()
        q, k, v, do = (torch.empty_like(t).copy_(t) for t in src)
        pause()
        o, lse = torch.zeros_like(q), torch.zeros((h, lead[0]) if packed else (lead[0], h, lead[1]), device="cuda")
        dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
        work = torch.full((layer.loco_attention_backward_workspace_bytes(q, k, **{x: y for x, y in kw.items() if packed}),), 255, dtype=torch.uint8, device="cuda")
        for _ in range(3):                           # each pass takes its operands from the one before
            layer.loco_attention_forward(q, k, v, o, lse, causal=True, **kw)
            pause()
            layer.loco_attention_backward(q, k, v, o, lse, do, dq, dk, dv, work, causal=True, **kw)
            pause()
            q, dq, k, dk, v, dv = dq, q, dk, k, dv, v
        return q, k, v, o, lse
    want = chain(torch.cuda.synchronize)
    for _ in range(10):
        got = chain(lambda: None)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))
    assert layer.loco_layer_status() == 0


@pytest.mark.parametrize("e,k", [(8, 2), (40, 3), (160, 6), (512, 16)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_router_backward_takes_an_index_out_of_range_as_no_choice(e, k, dtype):
    g = gen(43)
    z = normal(g, 70, e, dtype=dtype)
    cfg = layer.Router(e, k, normalize=False, balance_coef=0.3, z_coef=0.02)
    index, _, counts, _, _ = layer.router(z, cfg)
    dw, dl = torch.randn(70, k, generator=g, device="cuda"), torch.ones(2, device="cuda")
    none, wild = index.clone(), index.clone()
    none[::3, 0] = -1
    wild[::3, 0] = torch.tensor([e, e + 1, 1 << 30, -2, -(1 << 31), 600], device="cuda", dtype=torch.int32).repeat(4)
    want, got = torch.zeros(72, e, device="cuda", dtype=dtype), torch.zeros(72, e, device="cuda", dtype=dtype)
    layer.loco_router_backward(cfg, z, none, counts, want[1:71], dlosses=dl, dweights=dw)
    layer.loco_router_backward(cfg, z, wild, counts, got[1:71], dlosses=dl, dweights=dw)
    assert torch.equal(got, want) and not got[0].any() and not got[71].any() and bool(got[1:71].isfinite().all())


def test_a_wait_that_runs_out_ends_the_block_and_raises_the_flag(tmp_path):
    """Built into a library of its own, so that the flag of the one in use stays as it is."""
    here = os.path.dirname(os.path.abspath(__file__))
    lib = str(tmp_path / "wait.so")
    subprocess.check_call([loco_build.nvcc_path(), *loco_build.NVCC_FLAGS, "-shared", "-cudart", "static", "-o", lib, os.path.join(here, "attention_wait.cu")])
    L = ctypes.CDLL(lib)
    L.run_wait.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p]
    L.loco_layer_status.argtypes = [ctypes.POINTER(ctypes.c_uint32), ctypes.c_void_p]
    ns, flags, stream = torch.zeros(3, dtype=torch.int64, device="cuda"), ctypes.c_uint32(7), torch.cuda.current_stream().cuda_stream
    assert L.loco_layer_status(ctypes.byref(flags), stream) == 0 and flags.value == 0
    assert L.run_wait(ns.data_ptr(), 100, stream) == 0
    torch.cuda.synchronize()
    out, after, word = ns.tolist()
    assert 20_000_000 <= out < 1_000_000_000 and word == 1
    assert after < 2_000_000_000, "a hundred waits after it take less together than the limit of one"
    assert L.loco_layer_status(ctypes.byref(flags), stream) == 0 and flags.value == layer.FLAG_TIMEOUT
    assert layer.loco_layer_status() == 0


def run_attention(q, k, v, do, causal):
    b, s, h, _ = q.shape
    o, lse = torch.full_like(q, 7.0), torch.full((b, h, s), 7.0, device="cuda")
    layer.loco_attention_forward(q, k, v, o, lse, causal=causal)
    grads = [torch.full_like(t, 7.0) for t in (q, k, v)]
    work = torch.full((layer.loco_attention_backward_workspace_bytes(q, k),), 255, dtype=torch.uint8, device="cuda")
    layer.loco_attention_backward(q, k, v, o, lse, do, *grads, work, causal=causal)
    return (o, lse, *grads)


def positive_first(g, b, s, d):
    """Operands [b, s, 1, d] whose queries are positive, and at least 1/4, in the first dimension."""
    q, k, v, do = (normal(g, b, s, 1, d) for _ in range(4))
    q[..., 0] = q[..., 0].abs() + 0.25
    return q, k, v, do


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_with_an_infinite_score_is_nan_wherever_its_key_lies(d, causal):
    """Sample j has a score of +infinity at key j: o is NaN and lse +infinity for the queries that see it, and for no others."""
    n = 250
    q, k, v, do = positive_first(gen(51), n, n, d)
    plain = run_attention(q, k, v, do, causal)
    j = torch.arange(n, device="cuda")
    k[j, j, 0, 0] = math.inf
    o, lse, dq, dk, dv = run_attention(q, k, v, do, causal)
    sees = (j[None, :] >= j[:, None]) if causal else torch.ones(n, n, dtype=torch.bool, device="cuda")      # [sample, query]
    assert torch.equal(torch.isnan(o).all(-1).all(-1), sees) and torch.equal(torch.isnan(o).any(-1).any(-1), sees)
    assert torch.equal(lse[:, 0] == math.inf, sees) and torch.isfinite(lse[:, 0][~sees]).all()
    assert torch.isnan(dq[..., 1:])[sees].all() and torch.isnan(dv[j, j]).all()
    if causal:                       # two roundings of p and of o each
        off = (o.float() - plain[0].float()).abs().amax(-1)[..., 0][~sees]
        assert float(off.max()) <= 4 * U * float(v.float().abs().max())
        assert torch.isfinite(dq[~sees][..., 1:]).all()


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_key_with_a_score_of_minus_infinity_takes_no_part(d, causal):
    """Sample j has scores of -infinity at key j: p is zero there, as the 64-bit formulas have it."""
    n = 131
    q, k, v, do = positive_first(gen(52), n, n, d)
    j = torch.arange(n, device="cuda")
    k[j, j, 0, 0] = -math.inf
    o, lse, dq, dk, dv = run_attention(q, k, v, do, causal)
    for b in range(n):
        x, l, a = ref.attention(q[b, :, 0], k[b, :, 0], v[b, :, 0], causal, d ** -0.5)
        x = torch.nan_to_num(x)
        empty = l == -math.inf       # causal: the first query of sample 0 sees that key alone
        assert torch.equal(lse[b, 0][empty].double(), l[empty]) and int(empty.sum()) == (1 if causal and b == 0 else 0)
        assert float((lse[b, 0] - l)[~empty].abs().max()) <= 1e-4
        assert bool(((o[b, :, 0] - x).abs() <= U * x.abs() + (U + 1e-4) * a + 1e-30).all())
        want = ref.attention_gradient(q[b, :, 0], k[b, :, 0], v[b, :, 0], o[b, :, 0], lse[b, 0], do[b, :, 0], causal, d ** -0.5)
        for got, w, bound, dims in ((dq, want[0], want[3], slice(1, d)), (dk, want[1], want[4], slice(0, d)), (dv, want[2], want[5], slice(0, d))):
            w, bound = w[:, dims], bound[:, dims]
            assert bool(((got[b, :, 0, dims] - w).abs() <= U * w.abs() + (U + 1e-4) * bound + 2e-4 * (1 + float(bound.max()))).all())
        assert not dv[b, b].any() and not dk[b, b].any()


@pytest.mark.parametrize("d", [64, 128])
def test_attention_of_scores_that_are_all_minus_infinity_is_zero(d):
    q, k, v, do = positive_first(gen(53), 3, 200, d)
    k[1, :, 0, 0] = -math.inf
    o, lse, dq, dk, dv = run_attention(q, k, v, do, False)
    assert not o[1].any() and (lse[1] == -math.inf).all() and not dv[1].any() and not dk[1].any()
    for b in (0, 2):
        x, _, a = ref.attention(q[b, :, 0], k[b, :, 0], v[b, :, 0], False, d ** -0.5)
        assert bool(((o[b, :, 0] - x).abs() <= U * x.abs() + (U + 1e-4) * a + 1e-30).all())


@pytest.mark.parametrize("d", [64, 128])
def test_attention_query_that_is_nan_reaches_every_gradient_it_takes_part_in(d):
    """Sample i has a query i of NaN: its o, lse and dq are NaN, other queries' are not, and every key's dk and dv are."""
    n = 210
    q, k, v, do = positive_first(gen(54), n, n, d)
    i = torch.arange(n, device="cuda")
    q[i, i] = float("nan")
    o, lse, dq, dk, dv = run_attention(q, k, v, do, False)
    own = torch.eye(n, dtype=torch.bool, device="cuda")
    for t in (o, dq):
        bad = torch.isnan(t)[:, :, 0]
        assert torch.equal(bad.all(-1), own) and torch.equal(bad.any(-1), own)
    assert torch.equal(torch.isnan(lse[:, 0]), own)
    assert torch.isnan(dk).all() and torch.isnan(dv).all()


@pytest.mark.parametrize("n", [150, 128])
def test_attention_gradient_of_an_infinite_key_does_not_depend_on_where_the_queries_end(n):
    """All scores of key 3 are -infinity: no query takes it, whether or not a tile has rows past the last query."""
    for d in (64, 128):
        q, k, v, do = positive_first(gen(55), 1, n, d)
        k[0, 3, 0, 0] = -math.inf
        _, _, _, dk, dv = run_attention(q, k, v, do, False)
        assert not dk[0, 3].any() and not dv[0, 3].any() and bool(dk.isfinite().all()) and bool(dv.isfinite().all())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("e,k", [(8, 2), (16, 4), (40, 3), (65, 6), (160, 6), (256, 8), (512, 16)])
def test_router_counts_nan_as_infinity_in_the_choice(e, k, dtype):
    """Ties between the two go to the lowest expert; the losses are NaN."""
    z = normal(gen(61), 48, e, dtype=dtype)
    kind = torch.arange(48, device="cuda") % 6
    z[kind == 1, e - 2] = float("nan")
    z[kind == 2] = float("nan")
    z[kind == 3, 3], z[kind == 3, e - 3] = math.inf, float("nan")
    z[kind == 4, 1], z[kind == 4, e - 1] = float("nan"), math.inf
    z[kind == 5, ::2], z[kind == 5, 1::2] = math.inf, float("nan")
    # a NaN with its sign bit set and another payload
    bits = z.view(torch.int16 if dtype == BF else torch.int32)
    bits[1, e - 2] = -1
    index, _, counts, _, losses = layer.router(z, layer.Router(e, k, z_coef=1.0))
    order = torch.where(torch.isnan(z), math.inf, z.double()).cpu()
    want = torch.sort(order, dim=1, descending=True, stable=True)[1][:, :k]
    assert torch.equal(index.cpu().long(), want)
    assert torch.isnan(losses).all() and int(counts[e]) == 48
    assert torch.equal(counts[:e].cpu().long(), torch.bincount(want.flatten(), minlength=e))


@pytest.mark.parametrize("e", [9, 64, 65, 128, 160, 193, 256, 301, 512])
@pytest.mark.parametrize("k", [1, 3, 8, 9])
def test_router_choice_in_bfloat16(e, k):
    """Rows on which the choice can go wrong, a kind to a token; the order is that of the rounded logits."""
    g, n = gen(e * 17 + k), 700
    z = torch.randn(n, e, generator=g, device="cuda")
    kind, column = torch.arange(n, device="cuda") % 9, torch.arange(e, device="cuda")
    z = torch.where((kind == 1)[:, None], 0.25, z)                                     # all equal
    z = torch.where((kind == 2)[:, None], (z * 2).round() / 2, z)                      # few values, both zeros among them
    free = torch.rand(n, e, generator=g, device="cuda") < k * 1.2 / e
    z = torch.where((kind == 3)[:, None] & ~free, -math.inf, z)                        # about as many available as are chosen
    z = torch.where((kind == 4)[:, None], -math.inf, z)                                # none
    z = torch.where((kind == 5)[:, None] & (column > 0), torch.finfo(BF).min, z)
    z = torch.where((kind == 6)[:, None], column * 1e-3, z)                            # in order, ties by rounding
    z = torch.where((kind == 7)[:, None], column * -1e-3, z)
    z = torch.where((kind == 8)[:, None] & (column != e - 1), -math.inf, z).to(BF)
    index, _, counts, _, _ = layer.router(z, layer.Router(e, k))
    value, want = torch.sort(z.double().cpu(), dim=1, descending=True, stable=True)
    want = torch.where(value[:, :k] == -math.inf, -1, want[:, :k])
    assert torch.equal(index.cpu().long(), want)
    assert torch.equal(counts[:e].cpu().long(), torch.bincount(want[want >= 0], minlength=e))


def test_second_derivatives():
    """Rotary has them (against differentiation of its formula in 64 bits), attention and the router refuse them."""
    g = gen(71)
    table = torch.empty(30, 16, device="cuda")
    layer.loco_rotary_table(table, magnitude=1.2)
    q, k = normal(g, 2, 30, 3, 16, dtype=F32).requires_grad_(), normal(g, 2, 30, 1, 16, dtype=F32).requires_grad_()

    def second(y, x):
        grad, = torch.autograd.grad((y ** 3).sum() + (x ** 3).sum(), x, create_graph=True)
        return grad, torch.autograd.grad((grad ** 2).sum(), x)[0]
    x = q.detach().double().requires_grad_()
    c, s = table[:, None, :8].double(), table[:, None, 8:].double()
    plain = torch.cat([x[..., :8] * c - x[..., 8:] * s, x[..., 8:] * c + x[..., :8] * s], -1)
    for got, want in zip(second(layer.rotary(q, k, table)[0], q), second(plain, x)):
        # some twenty roundings in fp32 of terms that cancel to a tenth of their size at the least, in norm
        assert float((got.double() - want).detach().norm()) <= 200 * 2.0 ** -24 * float(want.detach().norm())
    heads = [normal(g, 1, 40, 2, 64).requires_grad_() for _ in range(3)]
    z = normal(g, 40, 8, dtype=F32).requires_grad_()
    for x, y in ((heads[0], layer.attention(*heads)), (z, layer.router(z, layer.Router(8, 2))[1])):
        grad, = torch.autograd.grad((y.float() ** 3).sum() + (x.float() ** 3).sum(), x, create_graph=True)
        with pytest.raises(RuntimeError, match="differentiated once"):
            torch.autograd.grad((grad.float() ** 2).sum(), x)


@pytest.mark.parametrize("how", ["plain", "lengths", "packed"])
def test_differentiable_attention_is_the_two_calls(how):
    """The same bits as loco_attention_forward and loco_attention_backward, with lengths and packed samples."""
    g, n = gen(72), [90, 0, 131]
    packed = how == "packed"
    lead = (sum(n),) if packed else (3, 131)
    q, k, v = (normal(g, *lead, h, 64).requires_grad_() for h in (4, 2, 2))
    w = normal(g, *lead, 4, 64)
    lens = {}
    if how == "lengths":
        lens = dict(len_q=torch.tensor(n, device="cuda", dtype=torch.int32), len_k=torch.tensor([131, 5, 64], device="cuda", dtype=torch.int32))
    elif packed:
        cu = torch.tensor([0] + n, device="cuda").cumsum(0).to(torch.int32)
        lens = dict(cu_q=cu, cu_k=cu, max_q=131, max_k=131)
    o = layer.attention(q, k, v, causal=True, scale=0.2, **lens)
    got = torch.autograd.grad((o * w).sum(), (q, k, v))
    q, k, v = (t.detach() for t in (q, k, v))
    want, lse = torch.empty_like(q), torch.empty((4, lead[0]) if packed else (3, 4, 131), device="cuda")
    layer.loco_attention_forward(q, k, v, want, lse, causal=True, scale=0.2, **lens)
    grads = [torch.empty_like(t) for t in (q, k, v)]
    work = torch.empty(layer.loco_attention_backward_workspace_bytes(q, k, **{x: y for x, y in lens.items() if packed}), dtype=torch.uint8, device="cuda")
    layer.loco_attention_backward(q, k, v, want, lse, w, *grads, work, causal=True, scale=0.2, **lens)
    assert torch.equal(o, want) and all(torch.equal(a, b) for a, b in zip(got, grads))
    assert any(bool(t.any()) for t in got)


def test_arguments_that_are_neither_true_nor_false_are_refused_before_a_launch():
    g, many = gen(73), torch.zeros(2)
    q, o, lse = normal(g, 1, 4, 2, 64), torch.zeros(1, 4, 2, 64, device="cuda", dtype=BF), torch.zeros(1, 2, 4, device="cuda")
    table = torch.empty(4, 64, device="cuda")
    layer.loco_rotary_table(table)
    z = normal(g, 4, 8)
    before = layer.loco_layer_launch_count()
    for call in (lambda: layer.loco_attention_forward(q, q, q, o, lse, causal=many),
                 lambda: layer.loco_rotary_apply(table, q, None, o, None, inverse=many),
                 lambda: layer.router(z, layer.Router(8, 2, normalize=many), work=torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")),
                 lambda: layer._binding().rotary_apply(table, q, None, o, None, None, 0, False, "a stream")):
        with pytest.raises(ValueError):
            call()
    assert layer.loco_layer_launch_count() == before and not o.any()


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_of_expanded_operands(d, causal):
    """Keys and values shared by the batch or by the heads, queries by the batch: the same bits as of copies; an expanded
    operand's gradient, summed by autograd, is the sum of the copies'."""
    g, b, s, h = gen(81), 3, 150, 4
    src = dict(q=normal(g, 1, s, h, d), k=normal(g, 1, s, h, d), v=normal(g, b, s, 1, d), one=normal(g, 1, s, 1, d), row=normal(g, b, 1, h, d))
    shape = (b, s, h, d)
    for names in (("q", "k", "v"), ("q", "one", "k"), ("row", "v", "row")):
        ops = [src[x].clone().requires_grad_() for x in names]
        seen = [t.expand(shape) for t in ops]
        copies = [t.detach().contiguous().requires_grad_() for t in seen]
        assert any(0 in t.stride() for t in seen)
        w = normal(g, *shape)
        o, want = layer.attention(*seen, causal=causal), layer.attention(*copies, causal=causal)
        assert torch.equal(o, want)
        spread = torch.autograd.grad(want, copies, w)
        for got, each, t in zip(torch.autograd.grad(o, ops, w), spread, ops):
            assert torch.equal(got, each.sum_to_size(t.shape))


def test_rotary_and_router_of_expanded_operands():
    g = gen(82)
    table = torch.empty(40, 64, device="cuda")
    layer.loco_rotary_table(table)
    q, k = normal(g, 1, 40, 1, 64).expand(2, 40, 6, 64), normal(g, 2, 1, 2, 64).expand(2, 40, 2, 64)
    for a, b in zip(layer.rotary(q, k, table), layer.rotary(q.contiguous(), k.contiguous(), table)):
        assert torch.equal(a, b)
    z, cfg = normal(g, 1, 40).expand(33, 40), layer.Router(40, 3, z_coef=0.1)
    for a, b in zip(layer.router(z, cfg), layer.router(z.contiguous(), cfg)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("where", [torch.int32, torch.int64])
def test_differentiable_rotary_with_positions_and_without_keys(layout, where):
    g = gen(91)
    table = torch.empty(70, 24, device="cuda")
    layer.loco_rotary_table(table, magnitude=1.1)
    q, k = normal(g, 2, 30, 3, 32).requires_grad_(), normal(g, 2, 30, 1, 32).requires_grad_()
    at = torch.randint(0, 70, (2, 30), generator=g, device="cuda", dtype=where)
    y, z = layer.rotary(q, k, table, positions=at, layout=layout)
    w = normal(g, 2, 30, 3, 32)
    got, zero = torch.autograd.grad(y, (q, k), w, allow_unused=True)
    want_y, want = torch.empty_like(w), torch.empty_like(w)
    layer.loco_rotary_apply(table, q.detach(), None, want_y, None, positions=at, layout=layout)
    layer.loco_rotary_apply(table, w, None, want, None, positions=at, layout=layout, inverse=True)
    assert torch.equal(y, want_y) and torch.equal(got, want) and (zero is None or not zero.any())
    alone, none = layer.rotary(q, None, table, positions=at, layout=layout)
    assert none is None and torch.equal(alone, y) and torch.equal(torch.autograd.grad(alone, q, w)[0], want)


@pytest.mark.parametrize("e,dtype", [(8, BF), (160, F32)])
def test_router_mask_of_truth_values_is_one_of_bytes(e, dtype):
    """Both directions, in the differentiable form; the masked tokens' logits may hold anything."""
    g = gen(92)
    z = normal(g, 90, e, dtype=dtype)
    mask = torch.rand(90, generator=g, device="cuda") < 0.6
    z[~mask] = float("nan")
    cfg, results = layer.Router(e, 2, balance_coef=0.3, z_coef=0.1), []
    for m in (mask, mask.to(torch.uint8) * 5):
        x = z.clone().requires_grad_()
        index, weight, counts, mean, losses = layer.router(x, cfg, mask=m)
        grad, = torch.autograd.grad(losses.sum() + (weight * torch.arange(2, device="cuda")).sum(), x)
        results.append((index, weight, counts, mean, losses, grad))
        assert int(counts[e]) == int(mask.sum()) and (index[~mask] == -1).all() and not weight[~mask].any()
        assert bool(losses.isfinite().all()) and not grad[~mask].any() and bool(grad[mask].any(1).all())
    assert all(torch.equal(a, b) for a, b in zip(*results))
    for bad in (mask[:89], mask.float(), torch.ones(180, dtype=torch.bool, device="cuda")[::2]):
        with pytest.raises(ValueError):
            layer.router(z, cfg, mask=bad)


def test_training_stops_where_a_wait_has_run_out(monkeypatch):
    import sys
    monkeypatch.syspath_prepend(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    sys.modules.pop("decoder_layer_step", None)
    import decoder_layer_step
    how = dict(steps=1, workers=1, batch=1, seq=40, report=lambda *_: None)
    assert len(decoder_layer_step.run(**how)) == 1 and layer.loco_layer_status() == 0
    monkeypatch.setattr(layer, "loco_layer_status", lambda: layer.FLAG_TIMEOUT)
    with pytest.raises(RuntimeError, match="ran out"):
        decoder_layer_step.run(**how)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("e", [8, 40, 160, 512])
def test_router_token_whose_logits_are_all_the_lowest_value(e, dtype):
    """It takes part with equal probabilities; without a coefficient its z loss is zero, not zero times an overflow."""
    z = normal(gen(95), 12, e, dtype=dtype)
    z[5] = torch.finfo(dtype).min
    for coef, want in ((0.0, 0.0), (1e-3, math.inf)):            # lse^2 is 1e77 for that token
        x = z.clone().requires_grad_()
        index, weight, counts, mean, losses = layer.router(x, layer.Router(e, 2, balance_coef=0.3, z_coef=coef))
        assert index[5].tolist() == [0, 1] and weight[5].tolist() == [0.5, 0.5] and int(counts[e]) == 12
        assert math.isfinite(float(losses.detach()[0])) and float(losses.detach()[1]) == want
        grad, = torch.autograd.grad(losses[0] + weight[:, 0].sum(), x)
        assert bool(grad.isfinite().all())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("packed", [False, True])
def test_attention_without_queries_or_without_keys(d, packed):
    g, lead = gen(96), (lambda n: (n,) if packed else (1, n))
    for nq, nk in ((0, 30), (30, 0), (0, 0)):
        q, k, v = (normal(g, *lead(n), 2, d).requires_grad_() for n in (nq, nk, nk))
        cu = lambda n: torch.tensor([0, n], device="cuda", dtype=torch.int32)
        o = layer.attention(q, k, v, causal=True, **(dict(cu_q=cu(nq), cu_k=cu(nk), max_q=nq, max_k=nk) if packed else {}))
        assert o.shape == q.shape and not o.any()
        for t, grad in zip((q, k, v), torch.autograd.grad(o, (q, k, v), torch.ones_like(o))):
            assert grad.shape == t.shape and not grad.any()


def test_attention_from_a_thread_that_has_not_touched_the_device():
    """Autograd's own thread is one where the backward call is the first of a program: no context is bound to it yet."""
    import threading
    g = gen(97)
    q, k, v, do = (normal(g, 1, 40, 2, 64) for _ in range(4))
    o, lse, grads = torch.zeros_like(q), torch.zeros(1, 2, 40, device="cuda"), [torch.zeros_like(q) for _ in range(3)]
    work = torch.zeros(layer.loco_attention_backward_workspace_bytes(q, k), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    calls = (lambda: layer.loco_attention_forward(q, k, v, o, lse),
             lambda: layer.loco_attention_backward(q, k, v, o, lse, do, *grads, work))
    for call in calls:
        failed = []

        def run():
            try:
                call()
            except Exception as e:
                failed.append(e)
        t = threading.Thread(target=run)
        t.start()
        t.join()
        assert not failed, failed
    want = run_attention(q, k, v, do, False)
    assert all(torch.equal(a, b) for a, b in zip((o, lse, *grads), want))


def test_attention_gradient_as_the_first_backward_pass_of_a_program():
    import subprocess
    import sys
    code = ("import torch; from paper_2407_04480_b200 import layer; "
            "q = torch.ones(1, 16, 2, 64, device='cuda', dtype=torch.bfloat16).requires_grad_(); g = torch.ones_like(q); "
            "print(float(torch.autograd.grad(layer.attention(q, q.detach(), q.detach()), q, g)[0].abs().max()))")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    out = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=120)
    assert out.returncode == 0 and float(out.stdout) == 0.0, out.stderr[-500:]          # all keys alike


def test_differentiable_forms_are_captured_into_a_graph():
    """Forward and backward of the three forms in one graph, replayed on other inputs."""
    g = gen(98)
    table = torch.empty(200, 64, device="cuda")
    layer.loco_rotary_table(table)
    cfg = layer.Router(8, 2, balance_coef=0.1, z_coef=0.01)
    work = torch.zeros(layer.loco_router_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    q, k, v = (normal(g, 2, 200, h, 64).requires_grad_() for h in (4, 2, 2))
    w = normal(g, 256, 8, dtype=F32)

    def step():
        o = layer.attention(*layer.rotary(q, k, table), v, causal=True)
        _, weight, _, _, losses = layer.router(o.flatten(2).flatten(0, 1).float() @ w, cfg, work=work)
        return torch.autograd.grad(losses.sum() + (weight[:, 0] * o.float().mean((2, 3)).flatten()).sum(), (q, k, v))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(2):
        with torch.no_grad():
            for t in (q, k, v):
                t.copy_(normal(g, *t.shape))
        graph.replay()
        assert all(torch.equal(a, b) and bool(a.any()) for a, b in zip(got, step()))
