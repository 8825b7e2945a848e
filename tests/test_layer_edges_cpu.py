"""Host-side edges of the decoder-layer operators that need no GPU: sizes past every limit, and what the differentiable forms
hand to the kernels, which stand-ins in plain torch take the place of."""
import struct

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


def heads(batch=0, row=0, head=0):
    return struct.pack("@Pqqq", PTR, batch, row, head)


def attention_cfg(batch=1, hq=1, hk=1, sq=1, sk=1):
    return layer._ATTENTION.pack(batch, hq, hk, 64, 0, sq, sk, 0, 0, 0, 0.125, 0, 0)


@pytest.mark.parametrize("size", [dict(batch=1 << 16, hq=512, hk=512, sk=65 * 128), dict(batch=1 << 16, hq=512, hk=512, sq=65 * 128),
                                  dict(batch=1 << 16, hq=512, hk=512, sq=129 * 128),
                                  dict(batch=1 << 30, hq=1 << 30, hk=1 << 30, sq=1 << 12, sk=1 << 12),
                                  dict(batch=1 << 16, hq=1 << 16, hk=1)])
def test_attention_refuses_more_blocks_than_a_launch_holds_before_it_launches_any(size):
    """More than 2^31 blocks in one of the call's kernels alone, or more than 64 bits hold."""
    cfg, x, L = attention_cfg(**size), heads(8, 8, 8), layer.lib()
    before = layer.loco_layer_launch_count()
    # the workspace is a number here, large enough for any of these
    assert L.loco_attention_backward(cfg, x, x, x, x, PTR, x, x, x, x, PTR, (1 << 64) - 1, None) == loco.ERR_UNSUPPORTED
    tiles = -(-size.get("sq", 1) // 256)                 # the forward kernel's, of 256 queries
    if tiles * size["batch"] * size["hq"] >= 1 << 31:
        assert L.loco_attention_forward(cfg, x, x, x, x, PTR, None) == loco.ERR_UNSUPPORTED
    assert layer.loco_layer_launch_count() == before
