"""Norm, sorted experts, their products and the clipped gradient on the GPU against 64 bits.

Tolerances count roundings: half a step of the output's type, and for sums in fp32 the number of additions in a row times
2^-24 of the sum of the absolute terms."""
import math

import pytest
import torch

from paper_2407_04480_b200 import layer, loco
from tests import experts_reference as ref

pytestmark = pytest.mark.gpu

BF, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
STEP = 2.0 ** -24
DEV = "cuda"


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def normal(g, *shape, dtype=BF, sigma=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * sigma).to(dtype)


def within(got, want, terms, additions, dtype):
    """|got - want| <= half a step of the type + additions * 2^-24 of the absolute terms, nowhere NaN where want is not."""
    room = want.abs() * ref.half_step(dtype) * 1.0001 + terms * (additions * STEP) + 1e-38
    off = (got.double() - want).abs()
    assert torch.isfinite(got.double()).all()
    assert bool((off <= room).all()), (float((off / room).max()), int((off > room).sum()))


# ---- norm ------------------------------------------------------------------------------------

# a chain of 32 elements a thread, five steps of a warp, sixteen warps: 53 additions in a row; then a root, products
NORM_ADDITIONS = 64
NORM_SHAPES = [(1, 1), (1, 8), (3, 7), (5, 64), (70, 76), (9, 512), (33, 513), (4, 1367), (130, 1032), (2, 4096), (3, 5120), (2, 8192), (3, 8200),
               (2, 16384), (2, 16383), (0, 64), (700, 128),
               (3000, 513), (2500, 1367), (1300, 2040), (700, 4096), (9000, 72),      # several teams of threads to a block,
               (60000, 40), (20011, 129), (5000, 1024)]                               # and several rows one after the other to a team


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,dim", NORM_SHAPES)
@pytest.mark.parametrize("residual,weight", [(True, True), (False, True), (True, False)])
def test_norm(rows, dim, dtype, residual, weight):
    g = gen(rows * 7 + dim)
    x, r, w = normal(g, rows, dim, dtype=dtype), normal(g, rows, dim, dtype=dtype), normal(g, dim, dtype=dtype)
    y, h = torch.full_like(x, 7.0), torch.full_like(x, 7.0)
    layer.loco_norm_forward(x, y, weight=w if weight else None, residual=r if residual else None, total=h if residual else None, eps=1e-5)
    if residual:
        want = (x.double() + r.double()).to(dtype)
        assert torch.equal(h, want)
    else:
        h = x
    if rows == 0:
        return
    want, _ = ref.norm(h, w if weight else None, 1e-5)
    within(y, want, want.abs(), NORM_ADDITIONS, dtype)
    again = torch.empty_like(y)                      # the norm of the kept sum has the same bits
    layer.loco_norm_forward(h, again, weight=w if weight else None, eps=1e-5)
    assert torch.equal(y, again)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("block", [0, 128])
@pytest.mark.parametrize("rows,dim", [s for s in NORM_SHAPES if s[0]])
def test_norm_in_8_bits(rows, dim, dtype, block):
    g = gen(rows * 5 + dim)
    x, r, w = normal(g, rows, dim, dtype=dtype), normal(g, rows, dim, dtype=dtype), normal(g, dim, dtype=dtype)
    if dim > 300:
        w[130:260] = 0                               # a run of 128 columns that holds nothing
    y, h = torch.empty(rows, dim, dtype=E4M3, device=DEV), torch.empty_like(x)
    scale = torch.empty(rows, -(-dim // block) if block else 1, device=DEV)
    layer.loco_norm_forward(x, y, weight=w, residual=r, total=h, scale=scale, block=block)
    want, _ = ref.norm(h, w, 1e-5)
    s, q = ref.e4m3(want, block)
    assert float(((scale.double() - s).abs() / s).max()) <= (NORM_ADDITIONS + 2) * STEP
    # 8 bits: half a step is 2^-4 of a normal value, 2^-10 of the type's least steps below; on top what fp32 did to the value
    room = q.abs() * (2.0 ** -4 + (2 * NORM_ADDITIONS + 4) * STEP) + 2.0 ** -10
    assert bool(((y.double() - q).abs() <= room).all())
    assert float(y.float().abs().max()) <= 448.0


@pytest.mark.parametrize("block", [0, 128])
@pytest.mark.parametrize("size", [1e-37, 1e-30, 1e-3, 1e18])
def test_norm_in_8_bits_of_small_and_large_weights(block, size):
    """Below 448 * 2^-126 the scale is its least value; nothing overflows on the way.  Values that fp32 holds as subnormals are off
    by 2^-150, which over 2^-126 is less than the 8 bits' least half step."""
    g = gen(12)
    x, w = normal(g, 5, 300, dtype=F32), normal(g, 300, dtype=F32, sigma=size)
    y, scale = torch.empty(5, 300, dtype=E4M3, device=DEV), torch.empty(5, -(-300 // block) if block else 1, device=DEV)
    layer.loco_norm_forward(x, y, weight=w, scale=scale, block=block)
    s, q = ref.e4m3(ref.norm(x, w, 1e-5)[0], block)
    assert float(((scale.double() - s).abs() / s).max()) <= (NORM_ADDITIONS + 2) * STEP
    room = q.abs() * (2.0 ** -4 + (2 * NORM_ADDITIONS + 4) * STEP) + 2.0 ** -10
    assert bool(((y.double() - q).abs() <= room).all())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,dim", NORM_SHAPES)
@pytest.mark.parametrize("past,weight", [(True, True), (False, True), (True, False)])
def test_norm_gradient(rows, dim, dtype, past, weight):
    g = gen(rows * 3 + dim)
    h, dy, dt, w = normal(g, rows, dim, dtype=dtype), normal(g, rows, dim, dtype=dtype), normal(g, rows, dim, dtype=dtype), normal(g, dim, dtype=dtype)
    dx, dw = torch.full_like(h, 7.0), torch.full_like(w, 7.0)
    work = torch.full((layer.loco_norm_backward_workspace_bytes(dim, dtype),), 255, dtype=torch.uint8, device=DEV)
    kw = dict(weight=w if weight else None, dtotal=dt if past else None)
    layer.loco_norm_backward(h, dy, dx, work, dweight=dw, **kw)
    if rows == 0:
        assert not dw.any()
        return
    want, terms, gw, gterms = ref.norm_gradient(h, dy, w if weight else None, dt if past else None, 1e-5)
    within(dx, want, terms, 3 * NORM_ADDITIONS, dtype)
    within(dw, gw, gterms, rows + NORM_ADDITIONS, dtype)
    alone, again = torch.empty_like(dx), torch.empty_like(dw)
    layer.loco_norm_backward(h, dy, alone, **kw)     # without the weight's gradient, and a second time
    layer.loco_norm_backward(h, dy, dt, work, dweight=again, **kw)       # into the gradient past the norm
    assert torch.equal(dx, alone) and torch.equal(dw, again) and (not past or torch.equal(dx, dt))


def test_norm_gradient_is_that_of_differences():
    """fp32: a step of 2^-6 each way; the third derivative is what the differences miss, (2^-6)^2 of the values."""
    g = gen(3)
    h, dy, w = (normal(g, *s, dtype=F32) for s in ((3, 40), (3, 40), (40,)))
    dx, dw, work = torch.empty_like(h), torch.empty_like(w), torch.empty(layer.loco_norm_backward_workspace_bytes(40, F32), dtype=torch.uint8, device=DEV)
    layer.loco_norm_backward(h, dy, dx, work, weight=w, dweight=dw)

    def at(h, w):
        y = torch.empty_like(h)
        layer.loco_norm_forward(h, y, weight=w)
        return float((y.double() * dy.double()).sum())
    step, floor = 2.0 ** -6, 40 * 3 * 2.0 ** -22 * 2 ** 6
    for i in range(3):
        for j in range(0, 40, 5):
            e = torch.zeros_like(h)
            e[i, j] = step
            assert abs((at(h + e, w) - at(h - e, w)) / (2 * step) - float(dx[i, j])) <= floor + 40 * step * step
    for j in range(40):
        e = torch.zeros_like(w)
        e[j] = step
        assert abs((at(h, w + e) - at(h, w - e)) / (2 * step) - float(dw[j])) <= floor       # linear


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("dim", [96, 4096])
def test_norm_strides_alignment_and_places(dtype, dim):
    """Rows inside wider ones, off the 16-byte boundaries, repeated rows, outputs over their inputs."""
    g = gen(dim)
    w = normal(g, dim, dtype=dtype)
    big, more = normal(g, 21, dim + 9, dtype=dtype), normal(g, 21, 2 * dim, dtype=dtype)
    x, r = big[:, 3:3 + dim], more[:, dim:]
    plain, total = torch.empty(21, dim, dtype=dtype, device=DEV), torch.empty(21, dim, dtype=dtype, device=DEV)
    layer.loco_norm_forward(x.contiguous(), plain, weight=w, residual=r.contiguous(), total=total)
    out = torch.zeros(21, dim + 5, dtype=dtype, device=DEV)
    h = torch.empty_like(total)
    layer.loco_norm_forward(x, out[:, 1:1 + dim], weight=w, residual=r, total=h)
    for a, b in ((out[:, 1:1 + dim], plain),):       # another width of access sums in another order
        within(a, b.double(), b.double().abs(), 2 * NORM_ADDITIONS, dtype)
    assert torch.equal(h, total) and not out[:, 0].any() and not out[:, 1 + dim:].any()
    y = torch.empty_like(plain)
    layer.loco_norm_forward(x, y, weight=w, residual=r, total=x)          # the sum over x itself
    assert torch.equal(x, total)
    z = total.clone()
    layer.loco_norm_forward(z, z, weight=w)
    assert torch.equal(z, plain)
    one = normal(g, 1, dim, dtype=dtype)
    many, single = torch.empty(5, dim, dtype=dtype, device=DEV), torch.empty(1, dim, dtype=dtype, device=DEV)
    layer.loco_norm_forward(one.expand(5, dim), many, weight=w)
    layer.loco_norm_forward(one, single, weight=w)
    assert torch.equal(many, single.expand(5, dim))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,dim", [(3000, 200), (2500, 700), (1000, 2100)])
def test_norm_of_many_rows_that_share_no_boundaries(rows, dim, dtype):
    """In single elements: a base off the boundaries, widths of their own."""
    g = gen(dim)
    x, r, dy = (normal(g, rows, dim + k, dtype=dtype)[:, k:] for k in (1, 3, 5))
    w = normal(g, dim + 1, dtype=dtype)[1:]
    y, h = torch.empty(rows, dim, dtype=dtype, device=DEV), torch.empty(rows, dim, dtype=dtype, device=DEV)
    layer.loco_norm_forward(x, y, weight=w, residual=r, total=h)
    assert torch.equal(h, (x.double() + r.double()).to(dtype))
    want, _ = ref.norm(h, w, 1e-5)
    within(y, want, want.abs(), NORM_ADDITIONS, dtype)
    for block in (0, 128):
        q, scale = torch.empty(rows, dim, dtype=E4M3, device=DEV), torch.empty(rows, -(-dim // block) if block else 1, device=DEV)
        layer.loco_norm_forward(h[:, :], q, weight=w, scale=scale, block=block)
        s, exact = ref.e4m3(want, block)
        assert float(((scale.double() - s).abs() / s).max()) <= (NORM_ADDITIONS + 2) * STEP
        assert bool(((q.double() - exact).abs() <= exact.abs() * (2.0 ** -4 + (2 * NORM_ADDITIONS + 4) * STEP) + 2.0 ** -10).all())
    dx, dw = torch.empty_like(y), torch.empty_like(w)
    layer.loco_norm_backward(h, dy, dx, torch.empty(layer.loco_norm_backward_workspace_bytes(dim, dtype), dtype=torch.uint8, device=DEV), weight=w, dweight=dw, dtotal=r)
    want, terms, gw, gterms = ref.norm_gradient(h, dy, w, r, 1e-5)
    within(dx, want, terms, 3 * NORM_ADDITIONS, dtype)
    within(dw, gw, gterms, rows + NORM_ADDITIONS, dtype)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("k,dim", [(2, 200), (6, 130), (3, 1001), (1, 129), (1, 1001), (1, 70), (2, 150), (4, 203), (5, 2502), (1, 5120), (2, 1367)])
def test_moves_of_rows_that_share_no_boundaries(k, dim, dtype):
    g = gen(dim)
    t, e = 3000, 8
    _, place = sorted_by(choices(g, t, k, e, "holes"), e)
    x, back, weight = normal(g, t, dim + 1, dtype=dtype)[:, 1:], normal(g, t * k, dim + 3, dtype=dtype)[:, 3:], torch.rand(t, k, generator=g, device=DEV)
    rows = torch.full((t * k, dim + 1), 7.0, dtype=dtype, device=DEV)[:, 1:]
    layer.loco_experts_dispatch(x, place, rows)
    some = place >= 0
    assert torch.equal(rows[place[some].long()], x[torch.arange(t, device=DEV)[:, None].expand(-1, k)[some]])
    y = torch.empty(t, dim + 1, dtype=dtype, device=DEV)[:, 1:]
    layer.loco_experts_combine(back, place, y, weight=weight)
    want, terms = ref.combine(back, place, weight)
    within(y, want, terms, k + 1, dtype)
    dweight = torch.empty(t, k, device=DEV)
    layer.loco_experts_combine_backward(x, back, place, weight, rows, dweight)
    want, live, dw, terms = ref.combine_gradient(x, back, place, weight)
    within(rows[live], want[live], want[live].abs(), 1, dtype)
    within(dweight, dw, terms, dim // 4 + 16, F32)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_norm_of_values_that_are_not_finite(dtype):
    """They reach their own row only; in 8 bits the scale says so."""
    g = gen(9)
    x = normal(g, 6, 256, dtype=dtype)
    x[1, 3], x[2, 200], x[4] = math.nan, math.inf, 0.0
    y = torch.empty_like(x)
    layer.loco_norm_forward(x, y)
    assert torch.isnan(y[1]).all() and torch.isnan(y[2, 200]) and not y[4].any()
    assert torch.isfinite(y[[0, 3, 5]]).all()
    q, s = torch.empty(6, 256, dtype=E4M3, device=DEV), torch.empty(6, 2, device=DEV)
    layer.loco_norm_forward(x, q, scale=s, block=128)
    assert torch.isnan(s[1]).all() and torch.isnan(s[2, 1]) and torch.isfinite(s[[0, 3, 4, 5]]).all()
    assert torch.isfinite((q.float() * s.repeat_interleave(128, 1))[[0, 3, 4, 5]]).all() and not q.float()[4].any()


# ---- experts ---------------------------------------------------------------------------------

def choices(g, tokens, k, experts, how="spread"):
    if how == "one":                                 # all to one expert
        return torch.full((tokens, k), experts - 1, dtype=torch.int32, device=DEV)
    index = torch.randint(0, experts, (tokens, k), generator=g, device=DEV, dtype=torch.int32)
    if how == "holes":
        index[torch.rand(tokens, k, generator=g, device=DEV) < 0.3] = -1
        if tokens > 3:
            index[2] = torch.tensor([experts, 1 << 30, -(1 << 31), -7], device=DEV, dtype=torch.int32).repeat(k)[:k]
    return index


def sorted_by(index, experts):
    offsets, place = torch.full((experts + 1,), 77, dtype=torch.int32, device=DEV), torch.full_like(index, 77)
    work = torch.full((layer.loco_experts_sort_workspace_bytes(experts),), 255, dtype=torch.uint8, device=DEV)
    layer.loco_experts_sort(index, offsets, place, work)
    return offsets, place


@pytest.mark.parametrize("tokens,k,experts", [(0, 2, 8), (1, 1, 1), (1, 2, 8), (9, 2, 8), (63, 4, 60), (700, 2, 8), (1024, 2, 8), (1025, 2, 8), (5021, 6, 160),
                                              (20000, 2, 4), (3000, 16, 512), (40000, 8, 256)])
@pytest.mark.parametrize("how", ["spread", "holes", "one"])
def test_sort(tokens, k, experts, how):
    index = choices(gen(tokens + k), tokens, k, experts, how)
    offsets, place = sorted_by(index, experts)
    first, want = ref.sort(index, experts)
    assert torch.equal(offsets.cpu(), first) and torch.equal(place.cpu(), want)


MOVES = [(1, 1, 1, 8), (9, 2, 8, 4096), (70, 2, 4, 76), (33, 6, 160, 2040), (51, 16, 64, 100), (40, 3, 8, 7), (300, 4, 8, 64), (5, 8, 16, 5121), (2, 2, 4, 1),
         (5000, 6, 16, 520), (3000, 2, 8, 1032), (20000, 3, 8, 72), (5000, 2, 8, 515), (4000, 5, 16, 1001), (2500, 16, 64, 264), (6000, 1, 4, 2056), (700, 4, 8, 1004),
         (9000, 1, 8, 64), (5000, 1, 8, 101), (3000, 1, 64, 502), (4000, 1, 8, 768), (4000, 2, 8, 520), (4000, 2, 8, 502), (2000, 2, 8, 1367), (2000, 6, 8, 502)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tokens,k,experts,dim", MOVES)
def test_dispatch_and_combine(tokens, k, experts, dim, dtype):
    g = gen(tokens + dim)
    index = choices(g, tokens, k, experts, "holes")
    offsets, place = sorted_by(index, experts)
    used, total = int(offsets[-1]), tokens * k
    x, weight = normal(g, tokens, dim, dtype=dtype), torch.rand(tokens, k, generator=g, device=DEV)
    rows = torch.full((total, dim), 7.0, dtype=dtype, device=DEV)
    layer.loco_experts_dispatch(x, place, rows)
    some = place >= 0
    assert torch.equal(rows[place[some].long()], x[torch.arange(tokens, device=DEV)[:, None].expand(-1, k)[some]])
    assert (rows[used:] == 7.0).all()
    back = normal(g, total, dim, dtype=dtype)
    back[used:] = math.nan                           # rows that no choice has
    for by in (weight, None):
        y = torch.full_like(x, 7.0)
        layer.loco_experts_combine(back, place, y, weight=by)
        want, terms = ref.combine(back, place, by)
        within(y, want, terms, k + 1, dtype)
    dy = normal(g, tokens, dim, dtype=dtype)
    drows, dweight = torch.full((total, dim), 7.0, dtype=dtype, device=DEV), torch.full((tokens, k), 7.0, device=DEV)
    layer.loco_experts_combine_backward(dy, back, place, weight, drows, dweight)
    want, live, dw, terms = ref.combine_gradient(dy, back, place, weight)
    within(drows[live], want[live], want[live].abs(), 1, dtype)
    assert (drows[~live] == 7.0).all()
    within(dweight, dw, terms, dim // 4 + 16, F32)


def test_places_outside_the_rows_are_none():
    g = gen(2)
    x = normal(g, 4, 64)
    place = torch.tensor([[0, -1], [3, 1], [1 << 30, -(1 << 31)], [2, 4]], dtype=torch.int32, device=DEV)
    rows = torch.full((3, 64), 7.0, dtype=BF, device=DEV)
    layer.loco_experts_dispatch(x, place, rows)
    assert torch.equal(rows, x[[0, 1, 3]])
    y = torch.empty_like(x)
    layer.loco_experts_combine(rows, place, y)
    assert torch.equal(y, torch.where(torch.tensor([True, True, False, True], device=DEV)[:, None], x, torch.zeros_like(x)))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_moves_with_strides_and_off_the_boundaries(dtype):
    g = gen(8)
    t, k, e, d = 37, 2, 8, 96
    _, place = sorted_by(choices(g, t, k, e), e)
    wide = normal(g, t, d + 7, dtype=dtype)
    x = wide[:, 3:3 + d]
    space = torch.full((t * k, d + 3), 7.0, dtype=dtype, device=DEV)
    rows = space[:, 1:1 + d]
    layer.loco_experts_dispatch(x, place, rows)
    assert torch.equal(rows[place.long()], x[:, None].expand(-1, k, -1)) and (space[:, 0] == 7.0).all() and (space[:, 1 + d:] == 7.0).all()
    y, z = torch.empty(t, d, dtype=dtype, device=DEV), torch.empty(t, d, dtype=dtype, device=DEV)
    layer.loco_experts_combine(rows, place, y)
    layer.loco_experts_combine(rows.contiguous(), place, z)
    assert torch.equal(y, z)
    weight, grads = torch.rand(t, k, generator=g, device=DEV), []
    for from_x, from_rows in ((x, rows), (x.contiguous(), rows.contiguous())):
        out, dw = torch.empty(t * k, d, dtype=dtype, device=DEV), torch.empty(t, k, device=DEV)
        layer.loco_experts_combine_backward(from_x, from_rows, place, weight, out, dw)
        grads.append((out, dw))
    assert torch.equal(grads[0][0], grads[1][0])
    one = normal(g, 1, d, dtype=dtype).expand(t, d)  # a broadcast gradient
    layer.loco_experts_dispatch(one, place, rows)
    assert torch.equal(rows, one[:1].expand(t * k, d))


# ---- products --------------------------------------------------------------------------------

def offsets_of(loads, start=0):
    return torch.tensor([start] + loads, dtype=torch.int32).cumsum(0).to(torch.int32).to(DEV)


PRODUCTS = [([1], 8, 8), ([0], 64, 64), ([3, 0, 1], 64, 256), ([130], 72, 264), ([128, 256, 64], 128, 512), ([0, 5, 0, 700, 63, 0], 200, 328), ([2, 1, 1, 0, 2, 2, 0, 0], 512, 1032),
            ([64] * 20, 64, 128), ([33, 129, 1, 65, 127], 1000, 776), ([1] * 100, 136, 72), ([0, 0, 0], 64, 64), ([300, 2500], 264, 512), ([40] * 5, 328, 40000), ([40] * 5, 64, 2000), ([9, 60, 12], 200, 20000), ([1], 4096, 20000),
            ([100, 0, 31, 200, 257], 520, 1000), ([1000], 128, 256), ([1000], 120, 512), ([513, 255], 1000, 264), ([15, 17, 16, 1, 31, 33, 49, 47], 264, 264),
            ([(i * 97) % 900 + 300 for i in range(40)], 72, 264), ([i % 3 for i in range(512)], 64, 72), ([i % 150 for i in range(70)], 264, 136), ([600, 0, 513, 1024], 136, 520),
            ([600, 0, 513, 1024, 300], 264, 96), ([256, 255, 257, 64, 1], 136, 128), ([70, 80, 90], 72, 8), ([600, 31, 513], 96, 264), ([1100], 200, 40),
            ([0, 1, 0, 1], 14336, 264), ([5, 17, 1], 12568, 160), ([150, 0, 150], 8192, 120), ([31, 33], 1544, 1000), ([64, 128, 1], 3080, 72), ([700], 4096, 128)]


@pytest.mark.parametrize("loads,d_in,d_out", PRODUCTS)
@pytest.mark.parametrize("transposed", [False, True])
def test_product(loads, d_in, d_out, transposed):
    """Rows in front of the first expert and behind the last hold NaN; they are not read as numbers and not written."""
    g = gen(sum(loads) + d_in)
    e, n = len(loads), sum(loads)
    offsets = offsets_of(loads, 3)
    x = torch.full((n + 8, d_in), math.nan, dtype=BF, device=DEV)
    x[3:3 + n] = normal(g, n, d_in)
    w = normal(g, e, d_out, d_in) if transposed else normal(g, e, d_in, d_out)
    y = torch.full((n + 8, d_out), 7.0, dtype=BF, device=DEV)
    layer.loco_experts_product(x, w, offsets, y, transposed=transposed)
    want, terms, live = ref.product(x, w, offsets, transposed)
    within(y[live], want[live], terms[live], 2 * d_in, BF)
    assert (y[~live] == 7.0).all()
    assert layer.loco_layer_status() == 0


@pytest.mark.parametrize("loads,d_in,d_out", PRODUCTS)
def test_product_weights(loads, d_in, d_out):
    """Rows that belong to no expert hold NaN or infinities, which lie in the same tiles as the last rows of an expert."""
    g = gen(sum(loads) + d_out)
    e, n = len(loads), sum(loads)
    offsets = offsets_of(loads, 5)
    a, b = torch.full((n + 90, d_in), math.nan, dtype=BF, device=DEV), torch.full((n + 90, d_out), math.inf, dtype=BF, device=DEV)
    a[5:5 + n], b[5:5 + n] = normal(g, n, d_in), normal(g, n, d_out)
    dw = torch.full((e, d_in, d_out), 7.0, dtype=BF, device=DEV)
    layer.loco_experts_product_weights(a, b, offsets, dw)
    want, terms = ref.product_weights(a, b, offsets)
    within(dw, want, terms, 2 * max(loads) + 2, BF)
    assert all(not dw[i].any() for i in range(e) if loads[i] == 0)
    again = torch.empty_like(dw)
    layer.loco_experts_product_weights(a, b, offsets, again)
    assert torch.equal(dw, again)
    assert layer.loco_layer_status() == 0


def test_product_of_rows_that_are_not_finite_stays_with_them():
    g = gen(6)
    offsets = offsets_of([40, 50, 60])
    x, w = normal(g, 150, 136), normal(g, 3, 136, 200)
    y, z = torch.empty(150, 200, dtype=BF, device=DEV), torch.empty(150, 200, dtype=BF, device=DEV)
    layer.loco_experts_product(x, w, offsets, y)
    x[45, 7], x[88, 0], w[2, 3, 9] = math.nan, math.inf, math.nan
    layer.loco_experts_product(x, w, offsets, z)
    off = (y != z).nonzero()
    assert set(off[:, 0].tolist()) == {45, 88, *range(90, 150)} and bool((off[off[:, 0] >= 90][:, 1] == 9).all())
    dw, dv = torch.empty(3, 136, 200, dtype=BF, device=DEV), torch.empty(3, 136, 200, dtype=BF, device=DEV)
    layer.loco_experts_product_weights(x, y, offsets, dw)
    x[45, 7] = x[88, 0] = 0.0
    layer.loco_experts_product_weights(x, y, offsets, dv)
    assert torch.equal(dw[[0, 2]], dv[[0, 2]]) and not torch.isfinite(dw[1, 7]).any() and torch.isfinite(dw[1, 1:7]).all()


@pytest.mark.parametrize("offsets", [[0, 10, 5, 40], [40, 0, 40, 0], [7, 30, 2, 1 << 30], [-4, 10, 20, 30], [0, 20, 100, 200], [50, 60, 70, 80], [40, 40, 40, 40], [0, 0, 0, 0]])
def test_product_clamps_offsets(offsets):
    g = gen(7)
    o = torch.tensor(offsets, dtype=torch.int32, device=DEV)
    x, w, b = normal(g, 40, 64), normal(g, 3, 64, 72), normal(g, 40, 72)
    y, dw = torch.full((40, 72), 7.0, dtype=BF, device=DEV), torch.empty(3, 64, 72, dtype=BF, device=DEV)
    layer.loco_experts_product(x, w, o, y)
    want, terms, live = ref.product(x, w, o, False)
    within(y[live], want[live], terms[live], 128, BF)
    assert (y[~live] == 7.0).all()
    layer.loco_experts_product_weights(x, b, o, dw)
    want, terms = ref.product_weights(x, b, o)
    within(dw, want, terms, 82, BF)


@pytest.mark.parametrize("transposed", [False, True])
def test_product_strides(transposed):
    """Rows and matrices inside wider ones, a matrix that all experts share, a row that repeats, one row, one expert."""
    g = gen(11)
    offsets = offsets_of([20, 0, 45, 7])
    shape = (4, 144, 80) if transposed else (4, 80, 144)
    x, y = normal(g, 72, 176)[:, 16:96], torch.full((72, 160), 7.0, dtype=BF, device=DEV)
    w = normal(g, 4, shape[1] + 3, shape[2] + 24)[:, 1:1 + shape[1], 8:8 + shape[2]]
    layer.loco_experts_product(x, w, offsets, y[:, 8:152], transposed=transposed)
    want, terms, _ = ref.product(x, w, offsets, transposed)
    within(y[:, 8:152], want, terms, 160, BF)
    assert (y[:, :8] == 7.0).all() and (y[:, 152:] == 7.0).all()
    shared = w[:1].expand(4, -1, -1)
    out = torch.empty(72, 144, dtype=BF, device=DEV)
    layer.loco_experts_product(x, shared, offsets, out, transposed=transposed)
    want, terms, _ = ref.product(x, shared, offsets, transposed)
    within(out, want, terms, 160, BF)
    same = x[:1].expand(72, -1)
    layer.loco_experts_product(same, w, offsets, out, transposed=transposed)
    want, terms, _ = ref.product(same, w, offsets, transposed)
    within(out, want, terms, 160, BF)
    dw = torch.full((4, 83, 168), 7.0, dtype=BF, device=DEV)
    layer.loco_experts_product_weights(x, out, offsets, dw[:, 2:82, 8:152])
    want, terms = ref.product_weights(x, out, offsets)
    within(dw[:, 2:82, 8:152], want, terms, 92, BF)
    assert (dw[:, :2] == 7.0).all() and (dw[:, 82:] == 7.0).all() and (dw[:, :, :8] == 7.0).all() and (dw[:, :, 152:] == 7.0).all()


# ---- gradient --------------------------------------------------------------------------------

def clip(gradients, outputs, most):
    squares, norm = torch.empty(1, dtype=torch.float64, device=DEV), torch.empty(1, device=DEV)
    work = torch.zeros(layer.loco_gradient_squares_workspace_bytes(), dtype=torch.uint8, device=DEV)
    layer.loco_gradient_squares(gradients, squares, work)
    layer.loco_gradient_clip(gradients, outputs, squares, norm, most)
    assert not work[:256].any()
    return squares, norm


SIZES = [[1], [7], [0], [], [8, 0, 3, 100003], [16384, 16385, 1, 16383], [5] * 300, [3] * 1700, [2_000_003, 11, 70_001], [40_000_000]]


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: "%d of %d" % (len(s), sum(s)))
@pytest.mark.parametrize("types", [(BF,), (F32,), (BF, F32)])
@pytest.mark.parametrize("limit", [0.5, 2.0, 0.0])
def test_clip(sizes, types, limit):
    """Tensors one after the other in a flat buffer, so that most start off the 16-byte boundaries."""
    g = gen(len(sizes))
    flat = {t: normal(g, sum(sizes) + 1, dtype=t, sigma=1e-3) for t in types}
    out = {t: torch.full_like(f, 7.0) for t, f in flat.items()}
    at, grads, outs = 0, [], []
    for i, n in enumerate(sizes):
        t = types[i % len(types)]
        grads.append(flat[t][at:at + n])
        outs.append(out[t][at:at + n])
        at += n
    total = ref.squares(grads)
    most = limit * math.sqrt(total)
    squares, norm = clip(grads, outs, most)
    # groups of eight squares in fp32, the rest in fp64
    assert abs(float(squares) - total) <= 9 * STEP * total
    assert abs(float(norm) - math.sqrt(total)) <= 6 * STEP * math.sqrt(total)
    by = most / math.sqrt(total) if math.sqrt(total) > most else 1.0
    for x, y in zip(grads, outs):
        within(y, x.double() * by, (x.double() * by).abs(), 8, x.dtype)
        if by == 1.0:
            assert torch.equal(x, y)
    assert all((out[t][sum(sizes):] == 7.0).all() for t in types)
    kept = [x.clone() for x in grads]
    again, _ = clip(grads, grads, most)              # in place
    assert torch.equal(again, squares)
    assert all(torch.equal(x, y) for x, y in zip(grads, outs)) or by == 1.0 and all(torch.equal(x, y) for x, y in zip(grads, kept))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("size", [1e30, 1e19, 1e-18, 1e-30])
def test_squares_past_the_range_of_fp32(dtype, size):
    x = (torch.rand(10007, generator=gen(4), device=DEV) * size).to(dtype)
    x[::3] = 0
    total = ref.squares([x])
    squares, _ = clip([x], [torch.empty_like(x)], 1.0)
    assert abs(float(squares) - total) <= 9 * STEP * total


def test_clip_outputs_that_meet_the_boundaries_elsewhere():
    g = gen(5)
    x = [normal(g, 30011, dtype=t) for t in (BF, F32, BF)]
    space = [torch.full((30020,), 7.0, dtype=t.dtype, device=DEV) for t in x]
    y = [s[k:k + 30011] for s, k in zip(space, (1, 3, 8))]
    clip(x, y, 1.0)
    z = [torch.empty_like(t) for t in x]
    clip(x, z, 1.0)
    assert all(torch.equal(a, b) for a, b in zip(y, z))
    assert all((s[:k] == 7.0).all() and (s[k + 30011:] == 7.0).all() for s, k in zip(space, (1, 3, 8)))


@pytest.mark.parametrize("bad,want", [(math.nan, math.nan), (math.inf, math.inf), (-math.inf, math.inf)])
def test_clip_of_gradients_that_are_not_finite(bad, want):
    g = gen(5)
    x = [normal(g, 5000), normal(g, 300, dtype=F32)]
    x[1][17] = bad
    y = [torch.empty_like(t) for t in x]
    _, norm = clip(x, y, 1.0)
    assert math.isnan(want) and math.isnan(float(norm)) or float(norm) == want
    if math.isnan(want):
        assert all(torch.isnan(t).all() for t in y)
    else:                                            # scaled by zero
        assert torch.isnan(y[1][17]) and not y[0].any() and not y[1][18:].any()


# ---- together --------------------------------------------------------------------------------

def layer_pass(x, r, w, index, weight, w1, w2):
    """A run of the operators as a layer makes it; everything is allocated here."""
    t, k = index.shape
    h, y = torch.empty_like(x), torch.empty_like(x)
    layer.loco_norm_forward(x, y, weight=w, residual=r, total=h)
    offsets, place = torch.empty(w1.shape[0] + 1, dtype=torch.int32, device=DEV), torch.empty_like(index)
    layer.loco_experts_sort(index, offsets, place, torch.empty(layer.loco_experts_sort_workspace_bytes(w1.shape[0]), dtype=torch.uint8, device=DEV))
    rows = torch.zeros(t * k, x.shape[1], dtype=BF, device=DEV)
    layer.loco_experts_dispatch(y, place, rows)
    mid, back, out = torch.zeros(t * k, w1.shape[2], dtype=BF, device=DEV), torch.zeros_like(rows), torch.empty_like(x)
    layer.loco_experts_product(rows, w1, offsets, mid)
    layer.loco_experts_product(mid, w2, offsets, back)
    layer.loco_experts_combine(back, place, out, weight=weight)
    dback, dweight = torch.zeros_like(back), torch.empty_like(weight)
    layer.loco_experts_combine_backward(out, back, place, weight, dback, dweight)
    dw2, dmid = torch.empty_like(w2), torch.zeros_like(mid)
    layer.loco_experts_product_weights(mid, dback, offsets, dw2)
    layer.loco_experts_product(dback, w2, offsets, dmid, transposed=True)
    dw1, drows = torch.empty_like(w1), torch.zeros_like(rows)
    layer.loco_experts_product_weights(rows, dmid, offsets, dw1)
    layer.loco_experts_product(dmid, w1, offsets, drows, transposed=True)
    dy, dx, dw = torch.empty_like(y), torch.empty_like(x), torch.empty_like(w)
    layer.loco_experts_combine(drows, place, dy)
    layer.loco_norm_backward(h, dy, dx, torch.empty(layer.loco_norm_backward_workspace_bytes(x.shape[1]), dtype=torch.uint8, device=DEV), weight=w, dweight=dw, dtotal=out)
    grads = [dw, dw1, dw2]
    squares, norm = torch.empty(1, dtype=torch.float64, device=DEV), torch.empty(1, device=DEV)
    layer.loco_gradient_squares(grads, squares, torch.zeros(layer.loco_gradient_squares_workspace_bytes(), dtype=torch.uint8, device=DEV))
    clipped = [torch.empty_like(t) for t in grads]
    layer.loco_gradient_clip(grads, clipped, squares, norm, 1.0)
    return [h, y, offsets, place, rows, out, dweight, dx, norm, *clipped]


def inputs(seed, t=333, k=2, e=8, d=200, f=328):
    g = gen(seed)
    return [normal(g, t, d), normal(g, t, d), normal(g, d), choices(g, t, k, e, "holes"), torch.rand(t, k, generator=g, device=DEV),
            normal(g, e, d, f, sigma=d ** -0.5), normal(g, e, f, d, sigma=f ** -0.5)]


def test_calls_in_a_row_read_what_the_launch_before_wrote(monkeypatch):
    """Every operand comes from the launches right before; the results are those of calls with pauses."""
    given = inputs(1)
    for name in [n for n in dir(layer) if n.startswith("loco_experts") or n.startswith("loco_norm") or n.startswith("loco_gradient")]:
        call = getattr(layer, name)
        monkeypatch.setattr(layer, name, lambda *a, call=call, **k: (torch.cuda.synchronize(), call(*a, **k), torch.cuda.synchronize())[1])
    want = layer_pass(*given)
    monkeypatch.undo()
    for _ in range(10):
        got = layer_pass(*[t.clone() for t in given])
        assert all(torch.equal(a, b) for a, b in zip(want, got))
    assert layer.loco_layer_status() == 0


def test_on_other_streams_and_captured():
    given = inputs(2)
    want = layer_pass(*given)
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    results = []
    for s in (a, b, a, b):                           # two at once
        with torch.cuda.stream(s):
            results.append(layer_pass(*given))
    torch.cuda.synchronize()
    for got in results:
        assert all(torch.equal(x, y) for x, y in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = layer_pass(*given)
    other = inputs(3)
    fresh = layer_pass(*other)
    for new, expect in ((other, fresh), (inputs(2), want), (other, fresh)):
        for t, n in zip(given, new):
            t.copy_(n)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(expect, held))
    assert layer.loco_layer_status() == 0


def test_the_stream_argument_is_the_one_that_is_used():
    g, s = gen(3), torch.cuda.Stream()
    x, y = normal(g, 50, 128), torch.zeros(50, 128, dtype=BF, device=DEV)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        x.mul_(2)
    layer.loco_norm_forward(x, y, eps=0.1, stream=s)
    s.synchronize()
    want, _ = ref.norm(x, None, 0.1)
    within(y, want, want.abs(), NORM_ADDITIONS, BF)


@pytest.mark.parametrize("call", [
    lambda: layer.loco_norm_forward(torch.ones(2, 8, device=DEV), torch.ones(2, 8, device=DEV, dtype=BF)),
    lambda: layer.loco_norm_forward(torch.ones(2, 8, device=DEV), torch.ones(2, 8, device=DEV), residual=torch.ones(2, 8, device=DEV)),
    lambda: layer.loco_norm_forward(torch.ones(2, 8, device=DEV), torch.ones(2, 8, device=DEV), total=torch.ones(2, 8, device=DEV)),
    lambda: layer.loco_norm_forward(torch.ones(2, 8, device=DEV), torch.ones(1, 8, device=DEV).expand(2, 8)),
    lambda: layer.loco_norm_forward(torch.ones(2, 8, device=DEV), torch.ones(2, 8, device=DEV).to(E4M3)),
    lambda: layer.loco_norm_forward(torch.ones(2, 8, device=DEV), torch.ones(2, 8, device=DEV).to(E4M3), scale=torch.ones(2, 1, device=DEV), block=64),
    lambda: layer.loco_norm_forward(torch.ones(2, 8, device=DEV), torch.ones(2, 8, device=DEV), block=128),
    lambda: layer.loco_norm_forward(torch.ones(2, 16392, device=DEV), torch.ones(2, 16392, device=DEV)),
    lambda: layer.loco_norm_forward(torch.ones(2, 8), torch.ones(2, 8)),
    lambda: layer.loco_norm_forward(torch.ones(2, 8, device=DEV), torch.ones(2, 8, device=DEV), weight=torch.ones(9, device=DEV)),
    lambda: layer.loco_norm_backward(*[torch.ones(2, 8, device=DEV)] * 3, dweight=torch.ones(8, device=DEV)),
    lambda: layer.loco_norm_backward(*[torch.ones(2, 8, device=DEV)] * 3, torch.ones(8, device=DEV), dweight=torch.ones(8, device=DEV)),
    lambda: layer.loco_experts_sort(torch.zeros(2, 2, device=DEV), torch.zeros(9, device=DEV).int(), torch.zeros(2, 2, device=DEV).int(), torch.zeros(1 << 20, device=DEV)),
    lambda: layer.loco_experts_sort(torch.zeros(2, 2, device=DEV).int(), torch.zeros(9, device=DEV).int(), torch.zeros(2, 2, device=DEV).int(), torch.zeros(8, device=DEV)),
    lambda: layer.loco_experts_sort(torch.zeros(2, 17, device=DEV).int(), torch.zeros(9, device=DEV).int(), torch.zeros(2, 17, device=DEV).int(), torch.zeros(1 << 20, device=DEV)),
    lambda: layer.loco_experts_dispatch(torch.ones(2, 8, device=DEV), torch.zeros(2, 2, device=DEV).int(), torch.ones(4, 8, device=DEV, dtype=BF)),
    lambda: layer.loco_experts_dispatch(torch.ones(2, 8, device=DEV), torch.zeros(3, 2, device=DEV).int(), torch.ones(4, 8, device=DEV)),
    lambda: layer.loco_experts_dispatch(torch.ones(2, 8, device=DEV), torch.zeros(2, 2, device=DEV).int(), torch.ones(1, 8, device=DEV).expand(4, 8)),
    lambda: layer.loco_experts_combine(torch.ones(4, 8, device=DEV), torch.zeros(2, 2, device=DEV).int(), torch.ones(2, 8, device=DEV), weight=torch.ones(2, 3, device=DEV)),
    lambda: layer.loco_experts_combine_backward(torch.ones(2, 8, device=DEV), torch.ones(4, 8, device=DEV), torch.zeros(2, 2, device=DEV).int(), None, torch.ones(4, 8, device=DEV), torch.ones(2, 2, device=DEV)),
    lambda: layer.loco_experts_product(torch.ones(4, 8, device=DEV), torch.ones(2, 8, 8, device=DEV), torch.zeros(3, device=DEV).int(), torch.ones(4, 8, device=DEV)),
    lambda: layer.loco_experts_product(torch.ones(4, 12, device=DEV, dtype=BF), torch.ones(2, 12, 8, device=DEV, dtype=BF), torch.zeros(3, device=DEV).int(), torch.ones(4, 8, device=DEV, dtype=BF)),
    lambda: layer.loco_experts_product(torch.ones(4, 16, device=DEV, dtype=BF), torch.ones(2, 16, 8, device=DEV, dtype=BF), torch.zeros(4, device=DEV).int(), torch.ones(4, 8, device=DEV, dtype=BF)),
    lambda: layer.loco_experts_product(torch.ones(5, 20, device=DEV, dtype=BF)[:, 4:12], torch.ones(2, 8, 8, device=DEV, dtype=BF), torch.zeros(3, device=DEV).int(), torch.ones(5, 8, device=DEV, dtype=BF)),
    lambda: layer.loco_experts_product_weights(torch.ones(4, 8, device=DEV, dtype=BF), torch.ones(4, 8, device=DEV, dtype=BF), torch.zeros(3, device=DEV).int(), torch.ones(1, 8, 8, device=DEV, dtype=BF).expand(2, 8, 8)),
    lambda: layer.loco_gradient_squares(torch.ones(4, device=DEV), torch.zeros(1, device=DEV, dtype=torch.float64), torch.zeros(1 << 20, device=DEV)),
    lambda: layer.loco_gradient_squares([torch.ones(4, device=DEV).half()], torch.zeros(1, device=DEV, dtype=torch.float64), torch.zeros(1 << 20, device=DEV)),
    lambda: layer.loco_gradient_squares([torch.ones(4, 4, device=DEV).T[1:]], torch.zeros(1, device=DEV, dtype=torch.float64), torch.zeros(1 << 20, device=DEV)),
    lambda: layer.loco_gradient_squares([torch.ones(4, device=DEV)], torch.zeros(1, device=DEV), torch.zeros(1 << 20, device=DEV)),
    lambda: layer.loco_gradient_squares([torch.ones(4, device=DEV)], torch.zeros(1, device=DEV, dtype=torch.float64), torch.zeros(8, device=DEV)),
    lambda: layer.loco_gradient_clip([torch.ones(4, device=DEV)], [], torch.zeros(1, device=DEV, dtype=torch.float64), None, 1.0),
    lambda: layer.loco_gradient_clip([torch.ones(4, device=DEV)], [torch.ones(4, device=DEV)], torch.zeros(1, device=DEV, dtype=torch.float64), None, -1.0),
    lambda: layer.loco_gradient_clip([torch.ones(4, device=DEV)], [torch.ones(4, device=DEV)], torch.zeros(1, device=DEV, dtype=torch.float64), None, math.nan),
    lambda: layer.loco_gradient_clip([torch.ones(4, device=DEV)] * 2, [torch.ones(4, device=DEV)] * 2, torch.zeros(1, device=DEV, dtype=torch.float64), None, 1.0),
    lambda: layer.loco_gradient_clip(list(torch.ones(12, device=DEV).unfold(0, 8, 4)), list(torch.ones(12, device=DEV).unfold(0, 8, 4)),
                                     torch.zeros(1, device=DEV, dtype=torch.float64), None, 1.0),
])
def test_refusals(call):
    before = layer.loco_layer_launch_count()
    with pytest.raises((ValueError, loco.LocoError)):
        call()
    assert layer.loco_layer_launch_count() == before


# ---- differentiable forms --------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF, F32])
def test_norm_form(dtype):
    """Leading dimensions, an operand cut out of a wider one, a broadcast gradient, one that never comes."""
    g = gen(21)
    wide = normal(g, 3, 5, 144, dtype=dtype)
    x, r, w = wide[..., 8:136].requires_grad_(), normal(g, 3, 5, 128, dtype=dtype).requires_grad_(), normal(g, 128, dtype=dtype).requires_grad_()
    y, total = layer.norm(x, w, residual=r)
    assert torch.equal(total, (x.detach().double() + r.detach().double()).to(dtype))
    want, _ = ref.norm(total.detach().flatten(0, 1), w.detach(), 1e-5)
    within(y.detach().flatten(0, 1), want, want.abs(), NORM_ADDITIONS, dtype)
    dy, dt = normal(g, 3, 1, 128, dtype=dtype).expand(3, 5, 128), normal(g, 3, 5, 128, dtype=dtype)
    for gy, gt in ((dy, dt), (dy, None), (None, dt)):
        outs, grads = zip(*[(o, d) for o, d in ((y, gy), (total, gt)) if d is not None])
        dx, dr, dw = torch.autograd.grad(outs, (x, r, w), grads, retain_graph=True)
        flat = lambda t: None if t is None else t.flatten(0, 1)
        want, terms, gw, gterms = ref.norm_gradient(flat(total.detach()), flat(dy if gy is not None else torch.zeros_like(dt)), w.detach(), flat(gt), 1e-5)
        within(dx.flatten(0, 1), want, terms, 3 * NORM_ADDITIONS, dtype)
        within(dw, gw, gterms, 15 + NORM_ADDITIONS, dtype)
        assert torch.equal(dx, dr)


def expert_block(x, index, weight, w1, w2):
    offsets, place = layer.experts_sort(index, w1.shape[0])
    a, b = layer.experts_product(layer.dispatch(x, place, offsets), w1, offsets).chunk(2, -1)
    return layer.combine(layer.experts_product(torch.nn.functional.silu(a) * b, w2, offsets, transposed=True), place, offsets, weight)


def block_inputs(seed, t=217, d=136, f=88, e=8, k=2):
    g = gen(seed)
    index = choices(g, t, k, e, "holes")
    return [normal(g, t, d), index, torch.rand(t, k, generator=g, device=DEV), normal(g, e, d, 2 * f, sigma=d ** -0.5), normal(g, e, d, f, sigma=f ** -0.5)]


def test_expert_forms_against_64_bits():
    """Two products, a gate and the weighted sum in a row, and back: a dozen roundings to 16 bits, each 2^-8 of its value, on the way
    to every gradient; the norm of the difference stays within 12 * 2^-8."""
    x, index, weight, w1, w2 = block_inputs(31)
    x, weight, w1, w2 = (t.requires_grad_() for t in (x, weight, w1, w2))
    y = expert_block(x, index, weight, w1, w2)
    dy = normal(gen(32), *y.shape)
    got = torch.autograd.grad(y, (x, weight, w1, w2), dy)
    X, W, A, B = (t.detach().double().requires_grad_() for t in (x, weight, w1, w2))
    Y = torch.zeros(x.shape, dtype=torch.float64, device=DEV)
    for e in range(8):
        token, slot = torch.where(index == e)
        a, b = (X[token] @ A[e]).chunk(2, -1)
        Y = Y.index_add(0, token, (torch.nn.functional.silu(a) * b) @ B[e].T * W[token, slot, None])
    want = torch.autograd.grad(Y, (X, W, A, B), dy.double())
    for a, b in zip((y.detach(), *got), (Y.detach(), *want)):
        assert float((a.double() - b).norm()) <= 12 * 2.0 ** -8 * float(b.norm())
    none = (index < 0) | (index >= 8)
    assert not got[1][none].any() and not got[0][none.all(1)].any()


def test_forms_leave_nothing_undefined_behind_the_last_expert():
    """Memory that the allocator hands out holds NaN; what goes on with all rows, a bias' gradient for one, must not see it."""
    x, index, weight, w1, w2 = block_inputs(33)
    junk = [torch.full((1 << 22,), math.nan, device=DEV, dtype=BF) for _ in range(4)]
    del junk
    offsets, place = layer.experts_sort(index, 8)
    used = int(offsets[-1])
    assert used < index.numel()
    bias = torch.zeros(w1.shape[2], device=DEV, dtype=BF, requires_grad=True)
    x.requires_grad_()
    rows = layer.dispatch(x, place, offsets)
    mid = layer.experts_product(rows, w1, offsets) + bias
    assert not rows[used:].any() and torch.isfinite(mid).all()
    y = layer.combine(layer.experts_product(mid.chunk(2, -1)[0].contiguous(), w2, offsets, transposed=True), place, offsets, weight)
    dx, db = torch.autograd.grad(y, (x, bias), torch.ones_like(y))
    assert torch.isfinite(dx).all() and torch.isfinite(db).all()


def test_forms_are_captured_into_a_graph():
    given = block_inputs(35)
    x, index, weight, w1, w2 = given
    leaves = [t.requires_grad_() for t in (x, weight, w1, w2)]
    scale = normal(gen(36), x.shape[1]).requires_grad_()

    def step():
        h, total = layer.norm(x, scale, residual=x.detach())
        grads = list(torch.autograd.grad((total + expert_block(h, index, weight, w1, w2)).float().square().mean(), [*leaves, scale]))
        norm = layer.clip_gradients(grads, 0.5, work=work)
        return [*grads, norm]
    work = torch.zeros(layer.loco_gradient_squares_workspace_bytes(), dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for seed in (37, 38):
        with torch.no_grad():
            for t, n in zip(given, block_inputs(seed)):
                t.copy_(n)
        graph.replay()
        assert all(torch.equal(a, b) and bool(a.any()) for a, b in zip(got, step()))


def test_clip_gradients_in_place():
    g = gen(41)
    grads = [normal(g, 7, 11), normal(g, 1001, dtype=F32), normal(g, 3)]
    kept = [t.clone() for t in grads]
    n = math.sqrt(ref.squares(kept))
    norm = layer.clip_gradients(grads, 2 * n)
    assert abs(float(norm) - n) <= 6 * STEP * n and all(torch.equal(a, b) for a, b in zip(grads, kept))
    layer.clip_gradients(grads, 0.25 * n)
    for a, b in zip(grads, kept):
        within(a, b.double() / 4, b.double().abs() / 4, 8, a.dtype)


def test_a_gradient_that_is_there_twice_is_refused_and_left_alone():
    x, work = torch.full((64,), 2.0, device=DEV), torch.zeros(layer.loco_gradient_squares_workspace_bytes(), dtype=torch.uint8, device=DEV)
    with pytest.raises(ValueError):
        layer.clip_gradients([x, torch.ones(3, device=DEV), x], 1.0, work=work)
    with pytest.raises(ValueError):
        layer.clip_gradients([x[:40], x[39:]], 1.0, work=work)
    assert (x == 2.0).all()
    layer.clip_gradients([x[40:], torch.ones(0, device=DEV), x[:40], x[:0]], 4.0, work=work)
    within(x, torch.full_like(x, 0.5), torch.full_like(x, 0.5), 4, F32)


def far(rows, dim, dtype=BF):
    """[rows, dim] whose last row lies past 2^32 elements, in a tensor of rows of 2^28."""
    space = torch.empty((rows - 1) * (1 << 28) + dim, dtype=dtype, device=DEV)
    return space.as_strided((rows, dim), (1 << 28, 1))


def test_rows_past_32_bits():
    g = gen(47)
    t, d = 18, 72
    x, y = far(t, d), far(t, d)
    x.copy_(normal(g, t, d))
    near = x.contiguous()
    layer.loco_norm_forward(x, y)
    want, dx, h = torch.empty_like(near), torch.empty_like(near), near.clone()
    layer.loco_norm_forward(near, want)
    assert torch.equal(y, want)
    layer.loco_norm_backward(x, x, y)
    layer.loco_norm_backward(near, near, dx)
    assert torch.equal(y, dx)
    place = torch.randperm(t, generator=g, device=DEV).int()[:, None]
    layer.loco_experts_dispatch(x, place, y)
    assert torch.equal(y[place[:, 0].long()], near)
    back = far(t, d)
    layer.loco_experts_combine(y, place, back)
    assert torch.equal(back, near)
    weight, dweight = torch.rand(t, 1, generator=g, device=DEV), torch.empty(t, 1, device=DEV)
    layer.loco_experts_combine_backward(x, y, place, weight, back, dweight)
    want, _, dw, terms = ref.combine_gradient(near, y.contiguous(), place, weight)
    within(back, want, want.abs(), 1, BF)
    within(dweight, dw, terms, d, F32)
    w, offsets = normal(g, 2, d, d), offsets_of([11, 7])
    layer.loco_experts_product(x, w, offsets, y)
    want, terms, _ = ref.product(near, w, offsets, False)
    within(y, want, terms, d, BF)
    layer.loco_experts_product_weights(x, y, offsets, w)
    want, terms = ref.product_weights(near, y.contiguous(), offsets)
    within(w, want, terms, 32, BF)
    layer.loco_experts_clear(y, offsets_of([16, 0]))
    assert y[:16].any(1).all() and not y[16:].any()
    assert torch.equal(h, near)


def test_a_gradient_past_32_bits():
    x = torch.zeros((1 << 32) + 11, dtype=BF, device=DEV)
    x[::1 << 24] = 3.0
    x[-1] = 4.0
    n = math.sqrt(257 * 9.0 + 16.0)
    norm = layer.clip_gradients([x], n / 2)
    assert abs(float(norm) - n) <= 2 * STEP * n
    assert float(x[-1]) == 2.0 and (x[::1 << 24] == 1.5).all() and int(x.count_nonzero()) == 258


def test_clear_zeroes_what_lies_behind_the_last_row():
    for dtype in (BF, F32):
        for last, dim in ((0, 5), (3, 130), (7, 64), (9, 64), (-5, 7)):
            rows = torch.full((7, dim + 3), 7.0, dtype=dtype, device=DEV)
            layer.loco_experts_clear(rows[:, 1:1 + dim], torch.tensor([0, 0, last], dtype=torch.int32, device=DEV))
            kept = min(max(last, 0), 7)
            assert (rows[:kept] == 7.0).all() and not rows[kept:, 1:1 + dim].any() and (rows[:, 0] == 7.0).all() and (rows[:, 1 + dim:] == 7.0).all()


def test_calls_from_a_thread_that_has_not_touched_the_device():
    import threading
    x, index, weight, w1, w2 = block_inputs(43)
    want = expert_block(x, index, weight, w1, w2)
    torch.cuda.synchronize()
    got, failed = [], []

    def run():
        try:
            got.append(expert_block(x, index, weight, w1, w2))
            torch.cuda.synchronize()
        except Exception as e:
            failed.append(e)
    t = threading.Thread(target=run)
    t.start()
    t.join()
    assert not failed, failed
    assert torch.equal(got[0], want)
