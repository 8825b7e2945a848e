"""Norm, sorted experts, their products and the clipped gradient where their ranges end: tiny values, offsets of every kind, lists that
overlap.  Tolerances count roundings, as in test_gpu_layer_experts.py."""
import math

import pytest
import torch

from paper_2407_04480_b200 import layer, loco
from tests import experts_reference as ref
from tests.test_gpu_layer_experts import BF, DEV, E4M3, F32, NORM_ADDITIONS, STEP, gen, normal

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
