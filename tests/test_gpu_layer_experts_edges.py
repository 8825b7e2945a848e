"""Norm, sorted experts, their products and the clipped gradient where their ranges end: tiny values, offsets of every kind, lists that
overlap.  Tolerances count roundings, as in test_gpu_layer_experts.py."""
import ctypes
import math
import os
import subprocess

import pytest
import torch

from paper_2407_04480_b200 import build as loco_build
from paper_2407_04480_b200 import layer
from tests import experts_reference as ref
from tests.test_gpu_layer_experts import BF, DEV, E4M3, F32, NORM_ADDITIONS, STEP, gen, normal, offsets_of, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("block", [0, 128])
@pytest.mark.parametrize("dim", [70, 300, 600, 4096])
@pytest.mark.parametrize("size", [1e-34, 1e-33, 1e-30, 1e-16])
def test_norm_in_8_bits_of_tiny_values_that_a_small_row_lifts(dim, block, dtype, size):
    """The largest |h w| of a run is about 3 h w: at 1e-33 times 1e-4 448 over it is past fp32's range, while the row's 1 / root mean square,
    about 300, keeps the scale above its least value.  A product of h and w that fp32 holds as a subnormal is off by 2^-150, which
    over a scale of 2^-126 is 2^-24, below the 8 bits' least half step."""
    g = gen(17)
    x, w = normal(g, 9, dim, dtype=dtype, sigma=1e-4), normal(g, dim, dtype=dtype, sigma=size)
    y, scale = torch.empty(9, dim, dtype=E4M3, device=DEV), torch.empty(9, -(-dim // block) if block else 1, device=DEV)
    layer.loco_norm_forward(x, y, weight=w, scale=scale, block=block)
    s, q = ref.e4m3(ref.norm(x, w, 1e-5)[0], block)
    assert bool(torch.isfinite(y.float()).all())
    # the scale's own rounding near its least value: a subnormal product's 2^-150 of 448 * 2^-126 is far below a step
    assert float(((scale.double() - s).abs() / s).max()) <= (NORM_ADDITIONS + 3) * STEP
    room = q.abs() * (2.0 ** -4 + (2 * NORM_ADDITIONS + 5) * STEP) + 2.0 ** -10
    assert bool(((y.double() - q).abs() <= room).all())


OFFSETS = [[0, 10, 5, 40], [40, 0, 40, 0], [7, 30, 2, 1 << 30], [-4, 10, 20, 30], [0, 20, 100, 200], [50, 60, 70, 80], [40, 40, 40, 40], [0, 0, 0, 0], [3, 9, 9, 25],
           [39, 39, 39, 39], [0, 30, 10, 20]]


@pytest.mark.parametrize("offsets", OFFSETS, ids=str)
def test_rows_of_no_expert_are_zeros_in_the_differentiable_product(offsets):
    """Offsets that do not begin with 0, or do not ascend, are read as the largest so far: the rows that this leaves to no expert are zeros
    in the outputs and in the gradient, and those of an expert are its products."""
    g = gen(51)
    junk = [torch.full((1 << 22,), math.nan, device=DEV, dtype=BF) for _ in range(4)]
    del junk
    o = torch.tensor(offsets, dtype=torch.int32, device=DEV)
    x, w, dy = normal(g, 40, 64).requires_grad_(), normal(g, 3, 64, 72), normal(g, 40, 72)
    y = layer.experts_product(x, w, o)
    dx, = torch.autograd.grad(y, x, dy)
    for got, (want, terms, live), n in ((y.detach(), ref.product(x.detach(), w, o, False), 64), (dx, ref.product(dy, w, o, True), 72)):
        within(got[live], want[live], terms[live], 2 * n, BF)
        assert not got[~live].any() and torch.isfinite(got).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("offsets", OFFSETS, ids=str)
def test_clear_others_zeroes_the_rows_of_no_expert_and_clear_those_from_the_last_offset_on(offsets, dtype):
    """The latter leaves alone what lies ahead: the rows of the experts before, where the offsets are a part of longer ones."""
    o = torch.tensor(offsets, dtype=torch.int32, device=DEV)
    others, behind = torch.ones(40, dtype=torch.bool), torch.arange(40) >= max(offsets[-1], 0)
    for a, b in ref.spans(o, 40):
        others[a:b] = False
    for call, zeros in ((layer.loco_experts_clear_others, others), (layer.loco_experts_clear, behind)):
        space = torch.full((40, 75), 7.0, dtype=dtype, device=DEV)
        rows = space[:, 1:74]
        call(rows, o)
        assert (rows[~zeros] == 7.0).all() and not rows[zeros].any() and (space[:, 0] == 7.0).all() and (space[:, 74] == 7.0).all()


def test_clear_others_with_as_many_experts_as_there_can_be():
    offsets = torch.arange(2, 515, dtype=torch.int32, device=DEV)     # 512 rows from the second on
    rows = torch.full((600, 8), 7.0, device=DEV)
    layer.loco_experts_clear_others(rows, offsets)
    assert not rows[:2].any() and (rows[2:514] == 7.0).all() and not rows[514:].any()


def _lists():
    x = torch.full((64,), 2.0, device=DEV)
    a, b = torch.ones(40, device=DEV), torch.ones(40, device=DEV)
    return {"swapped": ([a, b], [b, a]), "one in the other": ([x[:20], x[20:40]], [torch.empty(20, device=DEV), x[:20]]),
            "half of its own": ([x[:40]], [x[20:60]]), "ahead of its own": ([x[20:60]], [x[:40]]), "the last element": ([a, x[:25]], [x[24:], b[:25]]),
            "inside a larger one": ([x, a[:3]], [torch.empty(64, device=DEV), x[30:33]])}


@pytest.mark.parametrize("name", ["swapped", "one in the other", "half of its own", "ahead of its own", "the last element", "inside a larger one"])
def test_an_output_in_another_gradient_is_refused(name):
    gradients, outputs = _lists()[name]
    squares = torch.full((1,), 1e6, dtype=torch.float64, device=DEV)
    kept, before = [t.clone() for t in gradients], layer.loco_layer_launch_count()
    with pytest.raises(ValueError, match="overlap"):
        layer.loco_gradient_clip(gradients, outputs, squares, None, 1.0)
    assert layer.loco_layer_launch_count() == before and all(torch.equal(a, b) for a, b in zip(gradients, kept))


def test_outputs_beside_gradients_are_taken():
    x = torch.full((64,), 2.0, device=DEV)
    squares = torch.full((1,), 16.0, dtype=torch.float64, device=DEV)
    layer.loco_gradient_clip([x[:16], x[16:32], x[5:5]], [x[32:48], x[16:32], x[40:40]], squares, None, 1.0)
    assert x.tolist() == [2.0] * 16 + [0.5] * 32 + [2.0] * 16


def test_a_graph_notices_that_a_gradient_it_kept_has_been_clipped():
    x = torch.full((9,), 3.0, device=DEV, requires_grad=True)
    grad, = torch.autograd.grad((x ** 3).sum(), x, create_graph=True)
    kept = grad * grad                               # its backward pass needs the gradient as it was
    grad = grad.detach()
    version = grad._version
    norm = layer.clip_gradients([grad], 1.0)
    assert grad._version > version and float(norm) == pytest.approx(81.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        kept.sum().backward()


def test_gradients_without_a_version_are_clipped_all_the_same():
    with torch.inference_mode():
        grad = torch.full((4,), 2.0, device=DEV)
        layer.clip_gradients([grad], 1.0)
    assert grad.tolist() == [0.5] * 4


def test_a_wait_of_the_product_kernels_that_runs_out_raises_the_flag(tmp_path):
    """Built into a library of its own, with the attention kernels', so that the flags of the one in use stay as they are."""
    here, lib = os.path.dirname(os.path.abspath(__file__)), str(tmp_path / "wait.so")
    subprocess.check_call([loco_build.nvcc_path(), *loco_build.NVCC_FLAGS, "-shared", "-cudart", "static", "-o", lib,
                           os.path.join(here, "product_wait.cu"), os.path.join(here, "attention_wait.cu")])
    L = ctypes.CDLL(lib)
    L.run_product_wait.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p]
    L.loco_layer_status.argtypes = [ctypes.POINTER(ctypes.c_uint32), ctypes.c_void_p]
    ns, flags, stream = torch.zeros(3, dtype=torch.int64, device=DEV), ctypes.c_uint32(7), torch.cuda.current_stream().cuda_stream
    assert L.loco_layer_status(ctypes.byref(flags), stream) == 0 and flags.value == 0
    assert L.run_product_wait(ns.data_ptr(), 100, stream) == 0
    torch.cuda.synchronize()
    out, after, word = ns.tolist()
    assert 20_000_000 <= out < 1_000_000_000 and word == 1
    assert after < 2_000_000_000, "a hundred waits after it take less together than the limit of one"
    assert L.loco_layer_status(ctypes.byref(flags), stream) == 0 and flags.value == layer.FLAG_TIMEOUT
    assert layer.loco_layer_status() == 0


SKEWED = [([1200 if e == 20 else 4 + e % 3 for e in range(64)], 264, 520), ([0] * 100 + [1500] + [1] * 27, 520, 136), ([3000 if e == 0 else 0 for e in range(160)], 200, 72),
          ([2, 700, 1, 1], 1032, 264), ([5000] + [20] * 7, 264, 1000)]


@pytest.mark.parametrize("loads,d_in,d_out", SKEWED, ids=lambda v: "most %d" % max(v) if isinstance(v, list) else str(v))
@pytest.mark.parametrize("transposed", [False, True])
def test_products_of_one_expert_with_most_of_the_rows(loads, d_in, d_out, transposed):
    """The tiles' height goes by the average load, which says little here."""
    g = gen(sum(loads))
    n, e = sum(loads), len(loads)
    offsets = offsets_of(loads)
    x, b = normal(g, n, d_in), normal(g, n, d_out)
    w = normal(g, e, d_out, d_in) if transposed else normal(g, e, d_in, d_out)
    y, dw = torch.full((n, d_out), 7.0, dtype=BF, device=DEV), torch.full((e, d_in, d_out), 7.0, dtype=BF, device=DEV)
    layer.loco_experts_product(x, w, offsets, y, transposed=transposed)
    want, terms, _ = ref.product(x, w, offsets, transposed)
    within(y, want, terms, 2 * d_in, BF)
    layer.loco_experts_product_weights(x, b, offsets, dw)
    want, terms = ref.product_weights(x, b, offsets)
    within(dw, want, terms, 2 * max(loads) + 2, BF)
    assert layer.loco_layer_status() == 0


@pytest.mark.parametrize("loads,d_in,d_out", [([3, 0, 5], 4096, 1024), ([1] * 8, 1024, 2048), ([33, 129, 1, 65, 127], 1000, 776), ([700, 61, 1000, 0, 130], 520, 1000), ([64] * 30, 264, 264),
                                              ([127] * 40, 264, 520)])
def test_products_repeat_bit_for_bit_beside_other_work(loads, d_in, d_out):
    """The same inputs again, with another stream at the memory and calls close behind one another: every copy and product that an output
    depends on is waited for, or some repeat would differ."""
    g = gen(3)
    n, e = sum(loads), len(loads)
    offsets = offsets_of(loads)
    x, dy, w = normal(g, n, d_in), normal(g, n, d_out), normal(g, e, d_in, d_out)
    y, dx, dw = normal(g, n, d_out), torch.empty_like(x), torch.empty_like(w)

    def run():
        layer.loco_experts_product(x, w, offsets, y)
        layer.loco_experts_product(dy, w, offsets, dx, transposed=True)
        layer.loco_experts_product_weights(x, dy, offsets, dw)
    run()
    want = [t.clone() for t in (y, dx, dw)]
    junk, side = torch.zeros(1 << 26, dtype=torch.uint8, device=DEV), torch.cuda.Stream()
    for i in range(30):
        for t in (y, dx, dw):
            t.fill_(float(i))
        if i % 3:
            with torch.cuda.stream(side):
                for _ in range(8):
                    junk.add_(1)
        for _ in range(1 + i % 3):
            run()
        assert all(torch.equal(a, b) for a, b in zip((y, dx, dw), want)), i
    side.synchronize()
    assert layer.loco_layer_status() == 0


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n", [1, 32, 1000, 65_537, 4_000_001])
def test_squares_are_within_six_roundings(n, dtype):
    """bfloat16: a product of two is exact in fp32; three sums of a vector's pairs, one of the two halves, two of four vectors: six in a row.
    fp32: a product, a fused sum, the halves, four vectors: five.  All terms are positive, so that the bounds of the roundings add up to
    that of the sum; what comes in 64 bits after them is below 2^-40."""
    x = normal(gen(n), n, dtype=dtype, sigma=1e-3)
    squares, work = torch.empty(1, dtype=torch.float64, device=DEV), torch.zeros(layer.loco_gradient_squares_workspace_bytes(), dtype=torch.uint8, device=DEV)
    layer.loco_gradient_squares([x], squares, work)
    total = ref.squares([x])
    assert abs(float(squares) - total) <= (6 if dtype == BF else 5) * 1.00001 * STEP * total


def test_products_whose_contraction_is_shared_run_two_at_once_and_captured():
    """Few tiles: clusters of blocks share each, and leave their sums to one another.  On two streams at once, from a first call inside a
    capture, and replayed on other inputs."""
    given = [(normal(gen(s), 8, 4096), normal(gen(s + 1), 3, 4096, 1024)) for s in (61, 63)]
    offsets = offsets_of([3, 0, 5])
    outs = [[torch.empty(8, 1024, dtype=BF, device=DEV) for _ in range(20)] for _ in range(2)]
    graph, held = torch.cuda.CUDAGraph(), torch.empty(8, 1024, dtype=BF, device=DEV)
    x, w = (t.clone() for t in given[0])
    with torch.cuda.graph(graph):
        layer.loco_experts_product(x, w, offsets, held)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for i in range(20):
        for s, (a, b), out in zip(streams, given, outs):
            with torch.cuda.stream(s):
                layer.loco_experts_product(a, b, offsets, out[i])
    torch.cuda.synchronize()
    for (a, b), out in zip(given, outs):
        want, terms, _ = ref.product(a, b, offsets, False)
        within(out[0], want, terms, 2 * 4096, BF)
        assert all(torch.equal(out[0], o) for o in out)
        x.copy_(a), w.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(held, out[0])
    assert layer.loco_layer_status() == 0


def test_a_largest_norm_whose_conversion_changes_the_list():
    """The list is read after it: a number may be any object that converts to one."""
    gradients = [torch.full((4,), 2.0, device=DEV), torch.full((4,), 2.0, device=DEV)]
    outputs = [torch.empty(4, device=DEV), torch.empty(4, device=DEV)]

    class Limit:
        def __float__(self):
            gradients[1] = outputs[1] = None
            return 1.0
    before = layer.loco_layer_launch_count()
    with pytest.raises(ValueError, match="missing"):
        layer.loco_gradient_clip(gradients, outputs, torch.full((1,), 16.0, dtype=torch.float64, device=DEV), None, Limit())
    assert layer.loco_layer_launch_count() == before
