"""The decoder-layer operators on the GPU where they meet other work: launches in a row, values that are not finite, refusals."""
import ctypes
import math
import os
import subprocess

import pytest
import torch

from paper_2407_04480_b200 import build as loco_build
from paper_2407_04480_b200 import layer, loco

pytestmark = pytest.mark.gpu

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
