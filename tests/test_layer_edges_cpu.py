"""Host-side edges of the decoder-layer operators that need no GPU: sizes past every limit, and what the differentiable forms
hand to the kernels, which stand-ins in plain torch take the place of."""
import pytest
import torch

from paper_2407_04480_b200 import build as loco_build
from paper_2407_04480_b200 import layer, loco

PTR = 1 << 20                    # 16-byte aligned, never read


@pytest.fixture(scope="module", autouse=True)
def built():
    loco_build.build()


@pytest.mark.parametrize("tokens", [(1 << 31) // 4, 1 << 61, 1 << 62, (1 << 63) - 1])
def test_router_refuses_token_counts_whose_product_with_top_k_overflows(tokens):
    cfg = layer.Router(8, 4).c()
    L = layer.lib()
    assert L.loco_router_forward(cfg, tokens, PTR, 8, None, PTR, PTR, PTR, PTR, PTR, PTR, 1 << 30, None) == loco.ERR_ARG
    assert L.loco_router_backward(cfg, tokens, PTR, 8, None, PTR, PTR, None, None, PTR, 8, None) == loco.ERR_ARG
