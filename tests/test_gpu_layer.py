"""The decoder-layer operators on the GPU against plain 64-bit statements of their formulas.

Tolerances follow from the arithmetic: u = 2^-8 for every rounding to bfloat16 (relative to the rounded value; where
probabilities or their gradients are rounded before a product, relative to the sum of the product's absolute terms),
c * 2^-24 for c roundings in fp32."""
import math

import pytest
import torch

from paper_2407_04480_b200 import layer, loco
from tests import layer_reference as ref

pytestmark = pytest.mark.gpu

U, V = ref.U, 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(g, *shape, dtype=BF):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def close(got, want, bound, what=""):
    """got is within bound of want everywhere, and infinite exactly where want is."""
    got, want = got.double().cpu(), want.double().cpu()
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), what + ": infinities differ"
    assert not torch.isnan(got).any(), what + ": NaN"
    off = ((got - want).abs() - bound.double().cpu().broadcast_to(want.shape))[~inf]
    assert off.numel() == 0 or float(off.max()) <= 0, "%s: over the bound by %g at most" % (what, float(off.max()))


# ------------------------------------------------------------------------------------------------ rotary

@pytest.mark.parametrize("scaling", ["plain", "linear", "parts"])
@pytest.mark.parametrize("r,rows", [(2, 1), (64, 300), (128, 70001)])
def test_rotary_table(scaling, r, rows):
    t = torch.empty(rows, r, device="cuda")
    kw = dict(base=10000.0, scaling=scaling, factor=8.0, trained=4096.0, slow=1.0, fast=32.0, magnitude=1.25)
    layer.loco_rotary_table(t, **kw)
    # one rounding to fp32, and 64-bit angles of up to 7e4 radians in two libraries
    close(t, ref.rotary_table(rows, r, **kw), torch.full((1, 1), 1.25 * (V + 1e-10)), "table")


def check_rotary(b, s, hq, hk, d, r, layout, dtype, inverse, where, seed=1, fused=False, inplace=False):
    g = gen(seed)
    rows = s + 7
    table = torch.empty(rows, r, device="cuda")
    layer.loco_rotary_table(table, magnitude=1.1)
    if fused:
        x = normal(g, b, s, hq + 2 * hk, d, dtype=dtype)
        q, k = x[:, :, :hq], x[:, :, hq:hq + hk]
    else:
        q, k = normal(g, b, s, hq, d, dtype=dtype), normal(g, b, s, hk, d, dtype=dtype)
    pos = None
    if where:
        pos = torch.randint(0, rows, (b, s), generator=g, device="cuda", dtype=where)
    p = torch.arange(s).expand(b, s) if pos is None else pos
    want = [ref.rotary(t, table, p, layout, inverse) for t in (q, k)]
    size = [ref.rotary(t.abs(), table.abs(), p, "half" if layout == "half" else layout, False).abs() for t in (q, k)]
    outs = (q, k) if inplace else (torch.full_like(q, 9, memory_format=torch.contiguous_format), torch.full_like(k, 9, memory_format=torch.contiguous_format))
    sums = []
    for t in (q, k):               # |x_a c| + |x_b s| of every element
        y = t.double().abs().cpu()
        a = ref.rotary(y, table.abs(), p, layout, False)
        bb = ref.rotary(y, table.abs(), p, layout, True)
        sums.append(torch.maximum(a.abs(), bb.abs()))
    del size
    layer.loco_rotary_apply(table, q, k, *outs, positions=pos, layout=layout, inverse=inverse)
    for got, w, a in zip(outs, want, sums):
        close(got, w, 4 * V * a + (U * w.abs() if dtype == BF else 0), "rotary")
        if not inplace:
            assert got.shape == w.shape
    if r < d and not inplace:
        assert torch.equal(outs[0][..., r:], q[..., r:]), "dimensions past the rotated part are copied"


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,r", [(128, 128), (64, 16), (80, 32), (36, 10), (5, 4), (2, 2), (96, 96)])
def test_rotary_head_sizes(layout, dtype, d, r):
    check_rotary(2, 5, 3, 2, d, r, layout, dtype, False, torch.int32)
    check_rotary(1, 9, 4, 1, d, r, layout, dtype, True, None, fused=True)


@pytest.mark.parametrize("b,s,hq,hk", [(1, 1, 1, 1), (1, 1, 32, 8), (3, 67, 5, 3), (2, 1200, 32, 8)])
@pytest.mark.parametrize("where", [None, torch.int32, torch.int64])
def test_rotary_tokens_and_positions(b, s, hq, hk, where):
    check_rotary(b, s, hq, hk, 64, 64, "half", BF, False, where)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotary_in_place_equals_out_of_place_and_inverse_restores(layout):
    check_rotary(2, 33, 4, 2, 64, 32, layout, F32, False, torch.int64, inplace=True)
    check_rotary(2, 33, 4, 2, 64, 32, layout, BF, True, None, inplace=True, fused=True)


def test_rotary_misaligned_views_take_the_element_path():
    g = gen(5)
    table = torch.empty(16, 8, device="cuda")
    layer.loco_rotary_table(table)
    whole = normal(g, 1, 6, 3, 17)
    q = whole[..., 1:9]                              # two bytes past a boundary, odd strides
    out = torch.zeros(1, 6, 3, 8, device="cuda", dtype=BF)
    layer.loco_rotary_apply(table, q, None, out, None)
    want = ref.rotary(q, table, torch.arange(6)[None], "half", False)
    close(out, want, U * want.abs() + 8 * V * 4, "view")


def test_rotary_position_outside_the_table_gives_nan_in_the_rotated_part_only():
    g = gen(6)
    table = torch.empty(4, 8, device="cuda")
    layer.loco_rotary_table(table)
    q = normal(g, 1, 3, 2, 12)
    out = torch.zeros_like(q)
    layer.loco_rotary_apply(table, q, None, out, None, positions=torch.tensor([[-1, 2, 4]], device="cuda", dtype=torch.int32))
    assert torch.isnan(out[0, 0, :, :8]).all() and torch.isnan(out[0, 2, :, :8]).all()
    assert not torch.isnan(out[0, 1]).any() and torch.equal(out[..., 8:], q[..., 8:])


def test_rotary_gradient_is_the_transpose():
    """<y(x), w> = <x, y^T(w)> for random w, and the autograd form gives y^T(w)."""
    g = gen(7)
    table = torch.empty(64, 24, device="cuda")
    layer.loco_rotary_table(table, magnitude=1.3)
    q, k = (normal(g, 2, 50, h, 32, dtype=F32).requires_grad_() for h in (6, 2))
    for layout in ("half", "interleaved"):
        y, z = layer.rotary(q, k, table, layout=layout)
        wy, wz = normal(g, *y.shape, dtype=F32), normal(g, *z.shape, dtype=F32)
        gq, gk = torch.autograd.grad((y * wy).sum() + (z * wz).sum(), (q, k))
        a, b = float((y.detach().double() * wy.double()).sum()), float((q.detach().double() * gq.double()).sum())
        assert abs(a - b) <= 8 * V * float((y.detach().double() * wy.double()).abs().sum())
        # a broadcast gradient is given memory of its own
        y, z = layer.rotary(q, k, table, layout=layout)
        gq, = torch.autograd.grad(y.sum(), q)
        want = ref.rotary(torch.ones(2, 50, 6, 32), table, torch.arange(50).expand(2, 50), layout, True)
        close(gq, want, torch.full((1,), 8 * V * 2), "broadcast")


# ------------------------------------------------------------------------------------------------ attention

def samples(b, nq, nk, packed):
    """Per sample the places of its rows: (batch index or None, first, length)."""
    out, a, c = [], 0, 0
    for i in range(b):
        out.append(((None, a, nq[i]), (None, c, nk[i])) if packed else ((i, 0, nq[i]), (i, 0, nk[i])))
        a, c = a + nq[i], c + nk[i]
    return out


def rows(t, at, h):
    i, first, n = at
    return (t if i is None else t[i])[first:first + n, h]


def check_attention(b, sq, sk, hq, hk, d, causal, nq=None, nk=None, packed=False, seed=0, scale=None, views=None, spread=1.0):
    g = gen(seed + 17)
    ragged = nq is not None or nk is not None
    nq, nk = nq or [sq] * b, nk or [sk] * b
    if packed:
        sq, sk = sum(nq), sum(nk)
    lead_q, lead_k = ((sq,), (sk,)) if packed else ((b, sq), (b, sk))
    if views:
        q, k, v, do = views(g)
    else:
        q, do = normal(g, *lead_q, hq, d) * spread, normal(g, *lead_q, hq, d)
        k, v = normal(g, *lead_k, hk, d), normal(g, *lead_k, hk, d)
    lens = {}
    if packed:
        cu = lambda n: torch.tensor([0] + n, device="cuda").cumsum(0).to(torch.int32)
        lens = dict(cu_q=cu(nq), cu_k=cu(nk), max_q=max(nq + [0]), max_k=max(nk + [0]))
    elif ragged:
        lens = dict(len_q=torch.tensor(nq, device="cuda", dtype=torch.int32), len_k=torch.tensor(nk, device="cuda", dtype=torch.int32))
        for t, n in ((q, nq), (do, nq), (k, nk), (v, nk)):       # anything may lie past a sample's length
            for i in range(b):
                t[i, n[i]:] = float("nan")
                t[i, n[i]:n[i] + 1] = float("inf")
    o = torch.full(q.shape, 7.0, device="cuda", dtype=BF)
    lse = torch.full((hq, sq) if packed else (b, hq, sq), 7.0, device="cuda")
    layer.loco_attention_forward(q, k, v, o, lse, causal=causal, scale=scale, **lens)
    sc = scale if scale is not None else 1 / math.sqrt(d)
    want_o, want_l, bound = torch.zeros(q.shape, dtype=torch.float64), torch.full(lse.shape, -math.inf, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    at = samples(b, nq, nk, packed)
    for (aq, ak) in at:
        for h in range(hq):
            x, l, a = ref.attention(rows(q, aq, h), rows(k, ak, h // (hq // hk)), rows(v, ak, h // (hq // hk)), causal, sc)
            rows(want_o, aq, h)[:] = x.cpu()
            rows(bound, aq, h)[:] = a.cpu()
            (want_l[h] if packed else want_l[aq[0], h])[aq[1]:aq[1] + aq[2]] = l.cpu()
    # one rounding of p and one of o, the scores in fp32 (their terms' sizes are of order 30 at most here)
    close(o, want_o, U * want_o.abs() + (U + 1e-4 * max(1, spread)) * bound + 1e-30, "o")
    close(lse, want_l, 1e-4 * max(1, spread) * torch.ones(1), "lse")

    dq, dk, dv = (torch.full(t.shape, 7.0, device="cuda", dtype=BF) for t in (q, k, v))
    packed_kw = {x: lens[x] for x in ("cu_q", "cu_k", "max_q", "max_k") if x in lens}
    work = torch.full((layer.loco_attention_backward_workspace_bytes(q, k, **packed_kw),), 255, dtype=torch.uint8, device="cuda")
    layer.loco_attention_backward(q, k, v, o, lse, do, dq, dk, dv, work, causal=causal, scale=scale, **lens)
    wants = [torch.zeros(t.shape, dtype=torch.float64) for t in (q, k, v)]
    bounds = [torch.zeros(t.shape, dtype=torch.float64) for t in (q, k, v)]
    for (aq, ak) in at:
        for h in range(hq):
            j = h // (hq // hk)
            l = (lse[h] if packed else lse[aq[0], h])[aq[1]:aq[1] + aq[2]]
            r = ref.attention_gradient(rows(q, aq, h), rows(k, ak, j), rows(v, ak, j), rows(o, aq, h), l, rows(do, aq, h), causal, sc)
            for n, (a, head) in enumerate(((aq, h), (ak, j), (ak, j))):
                rows(wants[n], a, head)[:] += r[n].cpu()
                rows(bounds[n], a, head)[:] += r[3 + n].cpu()
    for name, got, w, a in zip(("dq", "dk", "dv"), (dq, dk, dv), wants, bounds):
        # ds = p (dp - D) loses up to 1e-4 of p times the sizes of dp and D, a few units here
        slack = 2e-4 * max(1, spread) * (1 + (float(a.max()) if a.numel() else 0.0))
        close(got, w, U * w.abs() + (U + 1e-4 * max(1, spread)) * a + slack, name)
    again = [torch.full(t.shape, 3.0, device="cuda", dtype=BF) for t in (q, k, v)]
    layer.loco_attention_backward(q, k, v, o, lse, do, *again, work, causal=causal, scale=scale, **lens)
    for x, y in zip((dq, dk, dv), again):
        assert torch.equal(x, y), "the same inputs give the same bits"


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("sq,sk", [(1, 1), (1, 300), (77, 77), (128, 128), (129, 129), (257, 255), (200, 130), (130, 200), (5, 0),
                                   (1, 65), (640, 64), (64, 640), (385, 511)])
def test_attention_lengths(sq, sk, causal):
    check_attention(1, sq, sk, 2, 2, 64, causal)
    check_attention(1, sq, sk, 4, 2, 128, causal, seed=1)


@pytest.mark.parametrize("d", [8, 16, 40, 64, 72, 96, 120, 128])
def test_attention_head_sizes(d):
    check_attention(2, 150, 150, 3, 3, d, True)
    check_attention(1, 70, 190, 4, 1, d, False)


@pytest.mark.parametrize("hq,hk", [(1, 1), (8, 1), (6, 3), (5, 5)])
def test_attention_shared_heads(hq, hk):
    check_attention(2, 140, 140, hq, hk, 64, True)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_padded_samples_with_garbage_past_their_length(causal, d):
    n = [150, 0, 1, 200, 64, 129]
    check_attention(6, 200, 200, 4, 2, d, causal, nq=n, nk=n)
    check_attention(4, 100, 300, 2, 2, d, causal, nq=[100, 3, 60, 0], nk=[7, 300, 0, 256])


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_packed_samples(causal, d):
    n = [1, 0, 130, 64, 257, 0, 3]
    check_attention(7, 0, 0, 4, 2, d, causal, nq=n, nk=n, packed=True)
    check_attention(3, 0, 0, 2, 2, d, causal, nq=[5, 128, 60], nk=[200, 1, 0], packed=True)


@pytest.mark.parametrize("d", [64, 128])
def test_attention_more_work_than_blocks_at_a_time(d):
    """Several hundred tiles of very different lengths, empty ones among them: a block takes up other blocks' work."""
    n = [300, 1, 0, 517, 128, 64, 0, 0, 255, 700, 3, 129, 400]
    check_attention(13, 0, 0, 24, 6, d, True, nq=n, nk=n, packed=True)
    check_attention(13, 700, 700, 16, 16, d, False, nq=n, nk=n)
    check_attention(3, 900, 500, 40, 8, d, True)


def test_attention_strided_operands():
    def fused(g):
        x = normal(g, 2, 150, 8, 64)
        return x[:, :, :4], x[:, :, 4:6], x[:, :, 6:], normal(g, 2, 150, 4, 64)

    def head_major(g):
        q, k, v, do = (normal(g, 2, h, 150, 64).transpose(1, 2) for h in (4, 2, 2, 4))
        return q, k, v, do

    def row_padded(g):
        return [normal(g, 2, 150, h, 88)[..., 8:72] for h in (4, 2, 2, 4)]
    for views in (fused, head_major, row_padded):
        check_attention(2, 150, 150, 4, 2, 64, True, views=views)


def test_attention_extreme_scores():
    check_attention(1, 130, 130, 2, 2, 64, True, spread=16.0)          # scores of hundreds: one key takes nearly all
    check_attention(1, 130, 130, 2, 2, 64, False, scale=0.0)           # all keys alike
    check_attention(1, 90, 90, 2, 2, 64, True, scale=-0.2)


def test_attention_long_row_and_many_tiles():
    check_attention(1, 2100, 2100, 2, 1, 128, True)
    check_attention(1, 3, 5000, 2, 1, 64, False)
    check_attention(1, 5000, 3, 2, 1, 64, False)


def test_attention_rows_beyond_32_bit_offsets():
    """Rows so far apart that the last ones lie past 2^31 elements."""
    big = torch.empty((1 << 31) + (1 << 25), dtype=BF, device="cuda")
    step = 1 << 24                                   # rows 128 and 129 start at 2^31 and beyond

    def views(g):
        out = []
        for i in range(4):
            t = big.as_strided((1, 130, 1, 64), (0, step, 64, 1), i * 4096) if i < 3 else normal(g, 1, 130, 1, 64)
            if i < 3:
                t.copy_(normal(g, 1, 130, 1, 64))
            out.append(t)
        return out
    check_attention(1, 130, 130, 1, 1, 64, True, views=views)
    del big
    torch.cuda.empty_cache()


def test_attention_on_another_stream():
    g = gen(3)
    q, k, v = (normal(g, 1, 500, 4, 64) for _ in range(3))
    o1, o2 = torch.empty_like(q), torch.empty_like(q)
    lse = torch.empty(1, 4, 500, device="cuda")
    layer.loco_attention_forward(q, k, v, o1, lse, causal=True)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        a = q * 2
        b = a / 2
        layer.loco_attention_forward(b, k, v, o2, lse, causal=True)
    s.synchronize()
    assert torch.equal(o1, o2)


def test_attention_gradient_against_differences():
    """<gradient, direction> against differences of sum(w o) along it, o by the 64-bit formula."""
    g = gen(11)
    q, k, v, w = (normal(g, 1, 100, 2, 64) for _ in range(4))
    for t in (q, k, v):
        t.requires_grad_()
    grads = torch.autograd.grad((layer.attention(q, k, v, causal=True) * w).sum(), (q, k, v))

    def value(*xs):
        return sum(float((ref.attention(*(x[0, :, h] for x in xs), True, 0.125)[0] * w[0, :, h].double()).sum()) for h in range(2))
    for i, grad in enumerate(grads):
        xs = [t.detach().double() for t in (q, k, v)]
        way = grad.detach().double() / grad.double().norm()      # the steepest one, so that the slope is not small by chance
        e = 1e-4
        up, down = list(xs), list(xs)
        up[i], down[i] = xs[i] + e * way, xs[i] - e * way
        slope = (value(*up) - value(*down)) / (2 * e)
        assert abs(slope - float((grad.double() * way).sum())) <= 4 * U * abs(slope)


def test_attention_refuses_wrong_tensors():
    g = gen(1)
    q = normal(g, 1, 4, 2, 64)
    o, lse = torch.empty_like(q), torch.empty(1, 2, 4, device="cuda")
    layer.loco_attention_forward(q, q, q, o, lse)
    for bad in (lambda: layer.loco_attention_forward(q.float(), q, q, o, lse),
                lambda: layer.loco_attention_forward(q, q, q[:, :3], o, lse),
                lambda: layer.loco_attention_forward(q, q, q, o, lse[:, :1]),
                lambda: layer.loco_attention_forward(q, q, q, o.transpose(2, 3), lse),
                lambda: layer.loco_attention_forward(q, q, q, o, lse, len_q=torch.zeros(1, device="cuda")),
                lambda: layer.loco_attention_forward(q[0], q[0], q[0], o[0], lse[0], cu_q=torch.zeros(2, device="cuda", dtype=torch.int32))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(loco.LocoError) as e:
        layer.loco_attention_forward(q[..., :60], q[..., :60], q[..., :60], o[..., :60], lse)
    assert e.value.code == loco.ERR_UNSUPPORTED
    with pytest.raises(loco.LocoError) as e:
        layer.loco_attention_forward(q[..., 4:60], q[..., 4:60], q[..., 4:60], o[..., 4:60], lse)
    assert e.value.code == loco.ERR_ALIGN


# ------------------------------------------------------------------------------------------------ router

def check_router(n, e, k, dtype, normalize, seed=0, mask=None, z=None, extra=0):
    g = gen(seed + 100)
    if z is None:
        whole = (torch.randn(n, e + extra, generator=g, device="cuda") * 1.5).to(dtype)
        z = whole[:, :e]
    cfg = layer.Router(e, k, normalize=normalize, balance_coef=0.3, z_coef=0.02)
    i, w = torch.full((n, k), 77, dtype=torch.int32, device="cuda"), torch.full((n, k), 7.0, device="cuda")
    c, m, l = torch.full((e + 1,), 77, dtype=torch.int32, device="cuda"), torch.full((e,), 7.0, device="cuda"), torch.full((2,), 7.0, device="cuda")
    work = torch.zeros(layer.loco_router_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    for _ in range(2):                                       # the workspace is left ready for the next call
        layer.loco_router_forward(cfg, z, i, w, c, m, l, work, mask=mask)
    zz = z.double().cpu().requires_grad_()
    ri, rw, rc, rm, rl = ref.router(zz, k, normalize, 0.3, 0.02, None if mask is None else mask.cpu())
    assert torch.equal(i.cpu(), ri) and torch.equal(c.cpu(), rc)
    # softmax and its sums: one fp32 rounding per step over e experts, the exponents' arguments of size up to 2 |z|
    top = float(z.double()[torch.isfinite(z)].abs().max()) if torch.isfinite(z).any() else 1.0
    eps = V * (e + 64 + 4 * top)
    close(w, rw.detach(), eps * rw.detach().abs() + 1e-37, "weight")
    close(m, rm.detach(), 2 * eps * rm.detach() + 1e-37, "mean")
    close(l, rl.detach(), 4 * eps * rl.detach().abs() + 1e-37, "losses")
    dw, dl = torch.randn(n, k, generator=g, device="cuda"), torch.tensor([1.7, -0.6], device="cuda")
    for use_l, use_w in ((True, True), (True, False), (False, True)):
        dz = torch.full_like(z, 7.0)
        layer.loco_router_backward(cfg, z, i, c, dz, mask=mask, dlosses=dl if use_l else None, dweights=dw if use_w else None)
        total = (rl * dl.double().cpu()).sum() * use_l + (rw * dw.double().cpu()).sum() * use_w
        want = torch.autograd.grad(total, zz, retain_graph=True)[0] if n and total.requires_grad else torch.zeros_like(zz)
        want = torch.where(torch.isinf(zz.detach()), 0.0, want)
        # every term is a probability times at most these sizes
        p = torch.where(torch.isinf(zz.detach()), 0.0, torch.softmax(torch.where(torch.isinf(zz.detach()), -1e30, zz.detach()), 1))
        act = max(int(rc[e]), 1)
        size = use_l * (0.3 * e * 1.7 * 2 / act + 0.02 * 2 * 0.6 * (top + math.log(e) + 1) / act)
        bound = eps * 4 * (p * size)
        if use_w:
            big = float(dw.abs().amax()) * (k + 1) if n else 0.0
            pw = p.clone()
            if normalize:                                    # a chosen weight may be much larger than its probability
                for t in range(n):
                    for j in range(k):
                        if ri[t, j] >= 0:
                            pw[t, ri[t, j].item()] = float(rw[t, j].detach())
            bound = bound + eps * 4 * big * pw
        close(dz, want, bound + (U * want.abs() if dtype == BF else 0) + 1e-37, "dlogits")


@pytest.mark.parametrize("e,k", [(1, 1), (2, 2), (7, 3), (8, 2), (16, 16), (13, 1), (17, 4), (32, 8), (33, 2), (64, 6), (100, 16), (160, 6), (256, 8), (257, 3), (512, 12)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_router_experts(e, k, dtype):
    for n in (1, 130):
        check_router(n, e, k, dtype, True, seed=e)
        check_router(n, e, k, dtype, False, seed=e + 1)


@pytest.mark.parametrize("e", [8, 40])
def test_router_masks_strides_and_ties(e):
    mask = (torch.rand(200, generator=gen(4), device="cuda") < 0.6).to(torch.uint8) * 3
    check_router(200, e, 2, BF, True, mask=mask)
    check_router(200, e, 2, F32, False, mask=torch.zeros(200, dtype=torch.uint8, device="cuda"))       # nobody takes part
    check_router(50, e, 4, F32, True, extra=3)                                                         # rows off every boundary
    check_router(50, e, 4, BF, True, extra=8)
    z = torch.randint(0, 2, (64, e), generator=gen(9), device="cuda").float()
    z[3] = 0.0
    z[5, ::2] = -0.0
    check_router(64, e, 3, F32, True, z=z)
    check_router(0, e, 2, F32, True)


@pytest.mark.parametrize("e", [8, 40])
def test_router_unavailable_experts_and_lowest_values(e):
    g = gen(12)
    z = torch.randn(40, e, generator=g, device="cuda")
    z[torch.rand(40, e, generator=g, device="cuda") < 0.7] = -math.inf
    z[7] = -math.inf                                          # an empty row
    z[8] = -math.inf
    z[8, e - 1] = 2.0                                         # one expert left
    check_router(40, e, 3, F32, True, z=z)
    z = torch.randn(20, e, generator=g, device="cuda")
    low = torch.finfo(F32).min
    z[torch.rand(20, e, generator=g, device="cuda") < 0.6] = low
    z[:, 1] = 0.5
    cfg = layer.Router(e, 3, z_coef=0.0)
    i, w, c, m, l = layer.router(z, cfg)
    ri, rw, rc, _, _ = ref.router(z.double().cpu(), 3, True, 0.01, 0.0)
    assert torch.equal(i.cpu(), ri) and torch.equal(c.cpu(), rc)
    close(w, rw, 1e-5 * rw + 1e-37, "weight")


def test_router_nan_is_loud():
    for e in (8, 40):
        z = torch.zeros(10, e, device="cuda")
        z[4, 2] = float("nan")
        i, w, c, m, l = layer.router(z, layer.Router(e, 2, z_coef=1.0))
        assert torch.isnan(l).all() and int(i[4, 0]) == 2 and int(c[e]) == 10
        assert int(i.min()) >= 0 and int(i.max()) < e


@pytest.mark.parametrize("e", [65, 128, 160, 190, 193, 256, 301, 512])
@pytest.mark.parametrize("k", [2, 3, 6, 8, 9, 16])
def test_router_choice_among_many_experts(e, k):
    """Rows on which the choice can go wrong, a kind to a token: most warps hold two kinds."""
    g, n = gen(e * 17 + k), 1500
    z = torch.randn(n, e, generator=g, device="cuda")
    kind = torch.arange(n, device="cuda") % 11
    z = torch.where((kind == 1)[:, None], 0.25, z)                                     # all equal
    z = torch.where((kind == 2)[:, None], (z * 2).round() / 2, z)                      # few values, both zeros among them
    free = torch.rand(n, e, generator=g, device="cuda") < k * 1.2 / e
    z = torch.where((kind == 3)[:, None] & ~free, -math.inf, z)                        # about as many available as are chosen
    z = torch.where((kind == 4)[:, None], -math.inf, z)                                # none
    near = torch.arange(e, device="cuda") % 64 < 4
    z = torch.where((kind == 5)[:, None] & near, z + 9, z)                             # the largest ones are one lane's
    z = torch.where((kind == 6)[:, None] & (torch.arange(e, device="cuda") > 0), torch.finfo(torch.float32).min, z)
    z = torch.where((kind == 7)[:, None], torch.arange(e, device="cuda") * 1e-3, z)    # in order
    z = torch.where((kind == 8)[:, None], torch.arange(e, device="cuda") * -1e-3, z)
    z = torch.where((kind == 9)[:, None] & (torch.arange(e, device="cuda") != e - 1), -math.inf, z)
    cfg = layer.Router(e, k)
    i, w, c, _, _ = layer.router(z, cfg)
    host = z.double().cpu()
    value, want = torch.sort(host, dim=1, descending=True, stable=True)
    value, want = value[:, :k], torch.where(value[:, :k] == -math.inf, -1, want[:, :k])
    assert torch.equal(i.cpu().long(), want)
    assert torch.equal(c[:e].cpu().long(), torch.bincount(want[want >= 0], minlength=e))
    p = torch.where(want >= 0, torch.exp(value - value[:, :1].clamp(min=-1e300)), 0.0)
    share = p.sum(1, keepdim=True)
    # exponents' arguments of size up to 2 |z| below the largest; what is further down than fp32 reaches is zero
    close(w, p / torch.where(share == 0, 1.0, share), V * (k + 16 + 64) * p + 1e-37, "weight")
    # a token's answer does not depend on its neighbours
    alone = z.clone()
    alone[kind != 0] = 0.25
    j, x, _, _, _ = layer.router(alone, cfg)
    assert torch.equal(j[kind == 0], i[kind == 0]) and torch.equal(x[kind == 0], w[kind == 0])


@pytest.mark.parametrize("e,k", [(160, 6), (512, 8)])
def test_router_nan_among_many_experts(e, k):
    z = torch.randn(40, e, generator=gen(3), device="cuda")
    z[4, e - 2] = float("nan")
    z[5, :] = float("nan")
    z[6, 3], z[6, e - 3] = math.inf, float("nan")
    i, _, _, _, l = layer.router(z, layer.Router(e, k, z_coef=1.0))
    assert torch.isnan(l).all() and int(i[4, 0]) == e - 2 and i[5].tolist() == list(range(k)) and i[6, :2].tolist() == [3, e - 3]
    rest = [t for t in range(40) if t not in (4, 5, 6)]
    assert torch.equal(i[rest].cpu().long(), torch.sort(z[rest].cpu(), dim=1, descending=True, stable=True)[1][:, :k])


def test_router_many_tokens_same_bits_twice():
    z = torch.randn(70001, 24, generator=gen(2), device="cuda") * 2
    cfg = layer.Router(24, 4, z_coef=0.1)
    a, b = layer.router(z, cfg), layer.router(z, cfg)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    p = torch.softmax(z.double(), 1)
    close(a[3], p.mean(0), 1e-5 * p.mean(0), "mean")
    assert int(a[2][:24].sum()) == 70001 * 4 and int(a[2][24]) == 70001


def test_router_gradient_against_differences():
    """Slope of (losses + weights) along the gradient, by differences of the forward kernel's own fp32 results."""
    g = gen(21)
    for e, k, normalize in ((8, 2, True), (48, 4, False)):
        z = (torch.randn(300, e, generator=g, device="cuda") * 2).requires_grad_()
        cfg = layer.Router(e, k, normalize=normalize, balance_coef=30.0, z_coef=3.0)
        dw = torch.randn(300, k, generator=g, device="cuda")

        def value(x):
            _, w, _, _, l = layer.router(x, cfg)
            return (w.double() * dw.double()).sum() + l.double().sum()
        grad, = torch.autograd.grad(value(z), z)
        way = grad / grad.norm()
        step = 2e-3
        with torch.no_grad():
            a, b = layer.router(z + step * way, cfg), layer.router(z - step * way, cfg)
            assert torch.equal(a[0], b[0]), "the choice must not change along the step"
            slope = float(value(z + step * way) - value(z - step * way)) / (2 * step)
        # differences lose 1e-7 of the values' size / step; third derivatives contribute step^2
        assert abs(slope - float(grad.norm())) <= 2e-3 * abs(slope) + 1e-6 * 300 / step


def test_calls_in_a_row_keep_the_streams_order():
    """Each call's kernels may be set up under the call before; every result has to be what calls with pauses give."""
    g = gen(31)
    b, s, h, hk, d = 2, 190, 4, 2, 64
    table = torch.empty(s, d, device="cuda")
    cfg = layer.Router(8, 2, z_coef=0.1)
    x = [normal(g, b, s, h, d), normal(g, b, s, hk, d), normal(g, b, s, hk, d)]
    proj = torch.randn(h * d, 8, generator=g, device="cuda").to(BF)

    def chain(pause):
        layer.loco_rotary_table(table, magnitude=1.1)
        pause()
        q, k = torch.zeros_like(x[0]), torch.zeros_like(x[1])
        layer.loco_rotary_apply(table, x[0], x[1], q, k)
        pause()
        o, lse = torch.zeros_like(q), torch.zeros(b, h, s, device="cuda")
        layer.loco_attention_forward(q, k, x[2], o, lse, causal=True)
        pause()
        z = o.reshape(b * s, h * d) @ proj
        i, w = torch.zeros(b * s, 2, dtype=torch.int32, device="cuda"), torch.zeros(b * s, 2, device="cuda")
        c, m, l = torch.zeros(9, dtype=torch.int32, device="cuda"), torch.zeros(8, device="cuda"), torch.zeros(2, device="cuda")
        work = torch.zeros(layer.loco_router_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
        layer.loco_router_forward(cfg, z, i, w, c, m, l, work)
        pause()
        dz = torch.zeros_like(z)
        layer.loco_router_backward(cfg, z, i, c, dz, dlosses=l, dweights=w)
        pause()
        do = (dz @ proj.T).view_as(o)
        dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(k)
        scratch = torch.zeros(layer.loco_attention_backward_workspace_bytes(q, k), dtype=torch.uint8, device="cuda")
        layer.loco_attention_backward(q, k, x[2], o, lse, do, dq, dk, dv, scratch, causal=True)
        pause()
        layer.loco_rotary_apply(table, dq, dk, dq, dk, inverse=True)
        layer.loco_rotary_apply(table, dq, dk, dq, dk)
        layer.loco_rotary_apply(table, dq, dk, dq, dk, inverse=True)
        return q, k, o, lse, z, i, w, c, m, l, dz, dq, dk, dv
    want = chain(torch.cuda.synchronize)
    for _ in range(20):
        got = chain(lambda: None)
        torch.cuda.synchronize()
        assert all(torch.equal(p, r) for p, r in zip(want, got))


def test_calls_are_captured_into_a_graph():
    g = gen(32)
    q, k, v, do = normal(g, 1, 300, 4, 64), normal(g, 1, 300, 2, 64), normal(g, 1, 300, 2, 64), normal(g, 1, 300, 4, 64)
    z, cfg = torch.randn(300, 8, generator=g, device="cuda"), layer.Router(8, 2)
    table = torch.empty(300, 64, device="cuda")
    layer.loco_rotary_table(table)
    o, lse = torch.empty_like(q), torch.empty(1, 4, 300, device="cuda")
    grads = [torch.empty_like(t) for t in (q, k, v)]
    scratch = torch.zeros(layer.loco_attention_backward_workspace_bytes(q, k), dtype=torch.uint8, device="cuda")
    i, w = torch.empty(300, 2, dtype=torch.int32, device="cuda"), torch.empty(300, 2, device="cuda")
    c, m, l = torch.empty(9, dtype=torch.int32, device="cuda"), torch.empty(8, device="cuda"), torch.empty(2, device="cuda")
    work = torch.zeros(layer.loco_router_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")

    def calls():
        layer.loco_attention_forward(q, k, v, o, lse, causal=True)
        layer.loco_attention_backward(q, k, v, o, lse, do, *grads, scratch, causal=True)
        layer.loco_rotary_apply(table, grads[0], grads[1], grads[0], grads[1], inverse=True)
        layer.loco_router_forward(cfg, z, i, w, c, m, l, work)
    calls()
    torch.cuda.synchronize()
    want = [t.clone() for t in (o, lse, *grads, i, w, c, m, l)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for t in (o, lse, *grads, w, m, l):
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (o, lse, *grads, i, w, c, m, l)))


def test_launches_are_counted():
    before = layer.loco_layer_launch_count()
    t = torch.empty(4, 8, device="cuda")
    layer.loco_rotary_table(t)
    assert layer.loco_layer_launch_count() == before + 1
