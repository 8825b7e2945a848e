"""Binding of the decoder-layer operators (include/loco_layer.h), and their differentiable forms.

The functions named loco_* have the name of the C entry point they call and only marshal arguments: every tensor,
outputs included, is the caller's, nothing is allocated and nothing synchronises.  `rotary`, `attention` and `router`
wrap them as torch.autograd functions that allocate their results.  All arithmetic runs in the CUDA kernels of
libloco_layer_b200.so; there is no CPU fallback: if the library cannot be loaded, the first call raises.
"""
from __future__ import annotations

import ctypes as C
import math
import os
import struct
from dataclasses import dataclass
from typing import Optional, Tuple

import torch

from .loco import BF16, F32, LocoError, OK, status_string

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libloco_layer_b200.so")

ROTARY_HALF, ROTARY_INTERLEAVED = 0, 1
ROTARY_PLAIN, ROTARY_LINEAR, ROTARY_PARTS = 0, 1, 2
LAYOUTS = {"half": ROTARY_HALF, "interleaved": ROTARY_INTERLEAVED}
SCALINGS = {"plain": ROTARY_PLAIN, "linear": ROTARY_LINEAR, "parts": ROTARY_PARTS}

EXPORTS = ("loco_rotary_table", "loco_rotary_apply", "loco_attention_forward", "loco_attention_backward",
           "loco_attention_backward_workspace_bytes", "loco_router_workspace_bytes", "loco_router_forward",
           "loco_router_backward", "loco_layer_status", "loco_layer_launch_count")
FLAG_TIMEOUT = 1

# the C structures, packed in one go: a call marshals a few dozen scalars and has to cost microseconds
_HEADS = struct.Struct("@Pqqq")                       # loco_heads_t
_TWO_HEADS = struct.Struct("@PqqqPqqq")
_TABLE = struct.Struct("@iiiffffff")                  # loco_rotary_table_t
_ROTARY = struct.Struct("@iiiiiiiii")                 # loco_rotary_t
_ATTENTION = struct.Struct("@iiiiiiiiiif4xPP")        # loco_attention_t
_ROUTER = struct.Struct("@iiiiff")                    # loco_router_t
_TWO_INTS = struct.Struct("@ii")

_lib = None


def lib() -> C.CDLL:
    """Load libloco_layer_b200.so (built by paper_2407_04480_b200.build); raises if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("LoCo layer library missing: %s (run python -m paper_2407_04480_b200.build); "
                               "there is no CPU fallback" % LIB_PATH)
        L = C.CDLL(LIB_PATH)
        u64, i64, i32, vp, st = C.c_uint64, C.c_int64, C.c_int32, C.c_void_p, C.c_char_p
        L.loco_rotary_table.argtypes = [st, vp, vp]
        L.loco_rotary_apply.argtypes = [st, vp, vp, st, st, st, i32, vp]
        L.loco_attention_forward.argtypes = [st] * 5 + [vp, vp]
        L.loco_attention_backward.argtypes = [st] * 5 + [vp] + [st] * 4 + [vp, u64, vp]
        L.loco_attention_backward_workspace_bytes.argtypes = [st]
        L.loco_router_workspace_bytes.argtypes = [st]
        L.loco_router_forward.argtypes = [st, i64, vp, i64, vp, vp, vp, vp, vp, vp, vp, u64, vp]
        L.loco_router_backward.argtypes = [st, i64, vp, i64, vp, vp, vp, vp, vp, vp, i64, vp]
        L.loco_layer_status.argtypes = [C.POINTER(C.c_uint32), vp]
        L.loco_layer_launch_count.argtypes = []
        for name in EXPORTS:
            getattr(L, name).restype = u64 if name.endswith(("_bytes", "_count")) else C.c_int
        _lib = L
    return _lib


def _check(code: int, where: str) -> None:
    if code != OK:
        raise LocoError(code, where)


# torch's accessor of the current stream's address; torch.cuda.current_stream() builds an object around it, which takes as
# long as a launch
_raw_stream = torch._C._cuda_getCurrentRawStream


def _stream(stream: Optional[torch.cuda.Stream], device: int) -> int:
    """The raw stream; the current device must be the operands' own, as for every call of the library."""
    if torch.cuda.current_device() != device:
        raise ValueError("the operands live on cuda:%d, which is not the current device" % device)
    return _raw_stream(device) if stream is None else stream.cuda_stream


def _dtype(t: torch.Tensor) -> int:
    if t.dtype is torch.bfloat16:
        return BF16
    if t.dtype is torch.float32:
        return F32
    raise ValueError("expected bfloat16 or float32, got %s" % t.dtype)


def _heads(t: torch.Tensor, shape, dtype, device: int) -> Tuple[int, int, int, int]:
    """(address, batch, row, head stride) of a [batch, row, head, dim] or [row, head, dim] tensor."""
    if t.dtype is not dtype or t.get_device() != device:
        raise ValueError("all heads must be %s on cuda:%d" % (dtype, device))
    if t.shape != shape:
        raise ValueError("expected heads of shape %s, got %s" % (tuple(shape), tuple(t.shape)))
    s = t.stride()
    if s[-1] != 1 and shape[-1] != 1:
        raise ValueError("the dimensions of a head must be contiguous")
    return (t.data_ptr(), s[0], s[1], s[2]) if len(s) == 4 else (t.data_ptr(), 0, s[0], s[1])


def _flat(t: Optional[torch.Tensor], shape, dtype, device: int, what: str) -> Optional[int]:
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != shape or t.get_device() != device or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor of shape %s on cuda:%d" % (what, dtype, tuple(shape), device))
    return t.data_ptr()


def loco_layer_launch_count() -> int:
    return int(lib().loco_layer_launch_count())


def loco_layer_status(stream=None) -> int:
    """Flags raised on the current device since the library was loaded; synchronises the stream."""
    flags = C.c_uint32(0)
    _check(lib().loco_layer_status(C.byref(flags), (torch.cuda.current_stream() if stream is None else stream).cuda_stream),
           "loco_layer_status")
    return int(flags.value)


# ---- rotary positions ------------------------------------------------------------------------

def loco_rotary_table(table: torch.Tensor, base: float = 10000.0, scaling: str = "plain", factor: float = 1.0,
                      trained: float = 4096.0, slow: float = 1.0, fast: float = 32.0, magnitude: float = 1.0,
                      stream=None) -> None:
    """Fill table (fp32 [positions, rotary_dim]): per position the cosines, then the sines of its pairs' angles."""
    if table.dim() != 2 or table.dtype != torch.float32 or not table.is_cuda or not table.is_contiguous():
        raise ValueError("expected a contiguous fp32 CUDA tensor [positions, rotary_dim]")
    if scaling not in SCALINGS:
        raise ValueError("scaling must be one of %s" % (tuple(SCALINGS),))
    cfg = _TABLE.pack(table.shape[1], table.shape[0], SCALINGS[scaling], base, factor, trained, slow, fast, magnitude)
    _check(lib().loco_rotary_table(cfg, table.data_ptr(), _stream(stream, table.get_device())), "loco_rotary_table")


def loco_rotary_apply(table: torch.Tensor, q: torch.Tensor, k: Optional[torch.Tensor], q_out: torch.Tensor,
                      k_out: Optional[torch.Tensor], positions: Optional[torch.Tensor] = None, layout: str = "half",
                      inverse: bool = False, stream=None) -> None:
    """Rotate q [batch, seq, heads, dim] into q_out and k (or None) into k_out; an output may be its input.

    table: from loco_rotary_table; positions: int32 or int64 [batch, seq], None for 0, 1, 2, ... in every sample."""
    kind = LAYOUTS.get(layout)
    if kind is None:
        raise ValueError("layout must be one of %s" % (tuple(LAYOUTS),))
    device, shape, dtype, tshape = q.get_device(), q.shape, q.dtype, table.shape
    if device < 0 or len(shape) != 4:
        raise ValueError("expected CUDA heads [batch, seq, heads, dim]")
    if table.dtype is not torch.float32 or len(tshape) != 2 or table.get_device() != device or not table.is_contiguous():
        raise ValueError("the table must be a contiguous fp32 tensor [positions, rotary_dim] on cuda:%d" % device)
    b, n, hq, d = shape
    hk = 0
    if k is None:
        xs, ys = _HEADS.pack(*_heads(q, shape, dtype, device)), _HEADS.pack(*_heads(q_out, shape, dtype, device))
    else:
        kshape = k.shape
        if len(kshape) != 4 or kshape[0] != b or kshape[1] != n or kshape[3] != d or k_out is None:
            raise ValueError("k must have q's batch, rows and head size, and an output")
        hk = kshape[2]
        xs = _TWO_HEADS.pack(*_heads(q, shape, dtype, device), *_heads(k, kshape, dtype, device))
        ys = _TWO_HEADS.pack(*_heads(q_out, shape, dtype, device), *_heads(k_out, kshape, dtype, device))
    at, wide = None, 0
    if positions is not None:
        if positions.dtype is torch.int32:
            wide = 4
        elif positions.dtype is torch.int64:
            wide = 8
        else:
            raise ValueError("positions must be int32 or int64")
        at = _flat(positions, (b, n), positions.dtype, device, "positions")
    cfg = _ROTARY.pack(_dtype(q), kind, d, tshape[1], b, n, tshape[0], wide, 1 if inverse else 0)
    _check(lib().loco_rotary_apply(cfg, table.data_ptr(), at, xs, ys, _TWO_INTS.pack(hq, hk), 1 if k is None else 2,
                                   _stream(stream, device)), "loco_rotary_apply")


# ---- attention -------------------------------------------------------------------------------

def _attention_config(q, k, causal, scale, len_q, len_k, cu_q, cu_k, max_q, max_k) -> Tuple[bytes, tuple]:
    """loco_attention_t and the shape of the log-sum-exp."""
    if not q.is_cuda or q.dtype is not torch.bfloat16:
        raise ValueError("attention takes bfloat16 CUDA tensors")
    packed = cu_q is not None or cu_k is not None
    device, qs, ks = q.get_device(), q.shape, k.shape
    if len(qs) != (3 if packed else 4) or len(ks) != len(qs) or ks[-1] != qs[-1]:
        raise ValueError("expected heads [batch, row, head, dim], or [row, head, dim] with cu_q and cu_k")
    if packed:
        if cu_q is None or cu_k is None or max_q is None or max_k is None or len_q is not None or len_k is not None:
            raise ValueError("packed samples need cu_q, cu_k, max_q and max_k and take no lengths")
        batch = cu_q.numel() - 1
        nq = _flat(cu_q, (batch + 1,), torch.int32, device, "cu_q")
        nk = _flat(cu_k, (batch + 1,), torch.int32, device, "cu_k")
        stats = (qs[1], qs[0])
    else:
        batch = qs[0]
        if ks[0] != batch:
            raise ValueError("queries and keys must have the same batch")
        nq = _flat(len_q, (batch,), torch.int32, device, "len_q")
        nk = _flat(len_k, (batch,), torch.int32, device, "len_k")
        max_q = max_k = 0
        stats = (batch, qs[2], qs[1])
    cfg = _ATTENTION.pack(batch, qs[-2], ks[-2], qs[-1], packed, qs[-3], ks[-3], max_q, max_k, 1 if causal else 0,
                          1.0 / math.sqrt(qs[-1]) if scale is None else scale, nq or 0, nk or 0)
    return cfg, stats


def loco_attention_forward(q, k, v, o, lse, causal: bool = False, scale: Optional[float] = None, len_q=None, len_k=None,
                           cu_q=None, cu_k=None, max_q: Optional[int] = None, max_k: Optional[int] = None, stream=None) -> None:
    """o = softmax(scale q k^T) v and the log-sum-exp of every row.

    Padded: q, o [batch, seq_q, heads, dim], k, v [batch, seq_k, heads_kv, dim], lse fp32 [batch, heads, seq_q], lengths
    len_q, len_k int32 [batch] (None: seq).  Packed: q, o [rows_q, heads, dim], k, v [rows_k, heads_kv, dim], lse
    [heads, rows_q], offsets cu_q, cu_k int32 [batch + 1], max_q, max_k the longest sample.  scale: None = 1/sqrt(dim)."""
    cfg, stats = _attention_config(q, k, causal, scale, len_q, len_k, cu_q, cu_k, max_q, max_k)
    dev, dt, qs, ks = q.get_device(), q.dtype, q.shape, k.shape
    _check(lib().loco_attention_forward(cfg, _HEADS.pack(*_heads(q, qs, dt, dev)), _HEADS.pack(*_heads(k, ks, dt, dev)),
                                        _HEADS.pack(*_heads(v, ks, dt, dev)), _HEADS.pack(*_heads(o, qs, dt, dev)),
                                        _flat(lse, stats, torch.float32, dev, "lse"), _stream(stream, dev)),
           "loco_attention_forward")


def loco_attention_backward_workspace_bytes(q, k, cu_q=None, cu_k=None, max_q=None, max_k=None) -> int:
    cfg, _ = _attention_config(q, k, False, None, None, None, cu_q, cu_k, max_q, max_k)
    return int(lib().loco_attention_backward_workspace_bytes(cfg))


def loco_attention_backward(q, k, v, o, lse, do, dq, dk, dv, work, causal: bool = False, scale: Optional[float] = None,
                            len_q=None, len_k=None, cu_q=None, cu_k=None, max_q: Optional[int] = None,
                            max_k: Optional[int] = None, stream=None) -> None:
    """dq, dk, dv from do and the forward pass's o and lse; arguments as loco_attention_forward.

    work: a contiguous CUDA tensor of loco_attention_backward_workspace_bytes() bytes or more."""
    cfg, stats = _attention_config(q, k, causal, scale, len_q, len_k, cu_q, cu_k, max_q, max_k)
    dev, dt, qs, ks = q.get_device(), q.dtype, q.shape, k.shape
    if work.get_device() != dev or not work.is_contiguous():
        raise ValueError("the workspace must be a contiguous tensor on cuda:%d" % dev)
    _check(lib().loco_attention_backward(cfg, _HEADS.pack(*_heads(q, qs, dt, dev)), _HEADS.pack(*_heads(k, ks, dt, dev)),
                                         _HEADS.pack(*_heads(v, ks, dt, dev)), _HEADS.pack(*_heads(o, qs, dt, dev)),
                                         _flat(lse, stats, torch.float32, dev, "lse"), _HEADS.pack(*_heads(do, qs, dt, dev)),
                                         _HEADS.pack(*_heads(dq, qs, dt, dev)), _HEADS.pack(*_heads(dk, ks, dt, dev)),
                                         _HEADS.pack(*_heads(dv, ks, dt, dev)), work.data_ptr(),
                                         work.numel() * work.element_size(), _stream(stream, dev)), "loco_attention_backward")


# ---- router ----------------------------------------------------------------------------------

@dataclass(frozen=True)
class Router:
    """Mirror of loco_router_t without the type of the logits, which is the tensor's own."""
    experts: int
    top_k: int
    normalize: bool = True
    balance_coef: float = 0.01
    z_coef: float = 0.0

    def c(self, dtype: int = BF16) -> bytes:
        return _ROUTER.pack(dtype, self.experts, self.top_k, 1 if self.normalize else 0, self.balance_coef, self.z_coef)


def loco_router_workspace_bytes(cfg: Router) -> int:
    return int(lib().loco_router_workspace_bytes(cfg.c()))


def _rows(t: torch.Tensor, cfg: Router, what: str) -> Tuple[int, int, int]:
    """(tokens, address, row stride) of a [tokens, experts] tensor."""
    shape = t.shape
    if not t.is_cuda or len(shape) != 2 or shape[1] != cfg.experts or (t.stride(1) != 1 and shape[1] > 1):
        raise ValueError("%s must be a CUDA tensor [tokens, %d] with contiguous rows" % (what, cfg.experts))
    return shape[0], t.data_ptr(), t.stride(0) if shape[0] > 1 else 0


def loco_router_forward(cfg: Router, logits, index, weight, counts, mean, losses, work, mask=None, stream=None) -> None:
    """Choice, weights, counts and losses of logits [tokens, experts]; see include/loco_layer.h for the outputs.

    work: a CUDA tensor of loco_router_workspace_bytes() bytes, zero before its first use."""
    n, at, stride = _rows(logits, cfg, "logits")
    dev, k = logits.get_device(), cfg.top_k
    if work.get_device() != dev or not work.is_contiguous():
        raise ValueError("the workspace must be a contiguous tensor on cuda:%d" % dev)
    _check(lib().loco_router_forward(cfg.c(_dtype(logits)), n, at, stride, _flat(mask, (n,), torch.uint8, dev, "mask"),
                                     _flat(index, (n, k), torch.int32, dev, "index"),
                                     _flat(weight, (n, k), torch.float32, dev, "weight"),
                                     _flat(counts, (cfg.experts + 1,), torch.int32, dev, "counts"),
                                     _flat(mean, (cfg.experts,), torch.float32, dev, "mean"),
                                     _flat(losses, (2,), torch.float32, dev, "losses"), work.data_ptr(),
                                     work.numel() * work.element_size(), _stream(stream, dev)), "loco_router_forward")


def loco_router_backward(cfg: Router, logits, index, counts, dlogits, mask=None, dlosses=None, dweights=None,
                         stream=None) -> None:
    """Gradient of the logits from those of the two losses (fp32 [2]) and of the weights (fp32 [tokens, top_k])."""
    n, at, stride = _rows(logits, cfg, "logits")
    dev, k = logits.get_device(), cfg.top_k
    n2, dat, dstride = _rows(dlogits, cfg, "dlogits")
    if n2 != n or dlogits.dtype != logits.dtype:
        raise ValueError("dlogits must have the logits' shape and type")
    _check(lib().loco_router_backward(cfg.c(_dtype(logits)), n, at, stride, _flat(mask, (n,), torch.uint8, dev, "mask"),
                                      _flat(index, (n, k), torch.int32, dev, "index"),
                                      _flat(counts, (cfg.experts + 1,), torch.int32, dev, "counts"),
                                      _flat(dlosses, (2,), torch.float32, dev, "dlosses"),
                                      _flat(dweights, (n, k), torch.float32, dev, "dweights"), dat, dstride,
                                      _stream(stream, dev)), "loco_router_backward")


# ---- differentiable forms --------------------------------------------------------------------

class _Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, table, positions, layout):
        ctx.save_for_backward(table, positions)
        ctx.layout = layout
        qo, ko = torch.empty_like(q, memory_format=torch.contiguous_format), torch.empty_like(k, memory_format=torch.contiguous_format)
        loco_rotary_apply(table, q, k, qo, ko, positions=positions, layout=layout)
        return qo, ko

    @staticmethod
    def backward(ctx, dq, dk):
        table, positions = ctx.saved_tensors
        dq, dk = dq.contiguous(), dk.contiguous()        # also a broadcast gradient gets memory of its own
        gq, gk = torch.empty_like(dq), torch.empty_like(dk)
        loco_rotary_apply(table, dq, dk, gq, gk, positions=positions, layout=ctx.layout, inverse=True)
        return gq, gk, None, None, None


def rotary(q, k, table, positions=None, layout: str = "half"):
    """Rotated queries and keys [batch, seq, heads, dim]."""
    return _Rotary.apply(q, k, table, positions, layout)


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, causal, scale, lens):
        lens = dict(lens)
        o = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        lse = torch.empty((q.shape[1], q.shape[0]) if lens.get("cu_q") is not None else (q.shape[0], q.shape[2], q.shape[1]),
                          dtype=torch.float32, device=q.device)
        loco_attention_forward(q, k, v, o, lse, causal=causal, scale=scale, **lens)
        ctx.save_for_backward(q, k, v, o, lse)
        ctx.how = (causal, scale, lens)
        return o

    @staticmethod
    def backward(ctx, do):
        q, k, v, o, lse = ctx.saved_tensors
        causal, scale, lens = ctx.how
        do = do.contiguous()
        dq, dk, dv = (torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k, v))
        packed = {x: lens.get(x) for x in ("cu_q", "cu_k", "max_q", "max_k")}
        work = torch.empty(loco_attention_backward_workspace_bytes(q, k, **packed), dtype=torch.uint8, device=q.device)
        loco_attention_backward(q, k, v, o, lse, do, dq, dk, dv, work, causal=causal, scale=scale, **lens)
        return dq, dk, dv, None, None, None


def attention(q, k, v, causal: bool = False, scale: Optional[float] = None, **lens):
    """softmax(scale q k^T) v; shapes and lengths as loco_attention_forward."""
    return _Attention.apply(q, k, v, causal, scale, lens)


class _Router(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, cfg, mask, work):
        n, dev = logits.shape[0], logits.device
        index = torch.empty((n, cfg.top_k), dtype=torch.int32, device=dev)
        weight = torch.empty((n, cfg.top_k), dtype=torch.float32, device=dev)
        counts = torch.empty(cfg.experts + 1, dtype=torch.int32, device=dev)
        mean, losses = torch.empty(cfg.experts, device=dev), torch.empty(2, device=dev)
        loco_router_forward(cfg, logits, index, weight, counts, mean, losses, work, mask=mask)
        ctx.save_for_backward(logits, index, counts, mask)
        ctx.cfg = cfg
        ctx.mark_non_differentiable(index, counts, mean)
        return index, weight, counts, mean, losses

    @staticmethod
    def backward(ctx, _index, dweight, _counts, _mean, dlosses):
        logits, index, counts, mask = ctx.saved_tensors
        dlogits = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
        loco_router_backward(ctx.cfg, logits, index, counts, dlogits, mask=mask, dlosses=dlosses.contiguous(),
                             dweights=dweight.contiguous())
        return dlogits, None, None, None


def router(logits, cfg: Router, mask=None, work: Optional[torch.Tensor] = None):
    """(index, weight, counts, mean, losses) of logits [tokens, experts]; weight and losses are differentiable.

    work: a workspace to keep between calls (loco_router_workspace_bytes() bytes, zeroed once); None allocates one."""
    if work is None:
        work = torch.zeros(loco_router_workspace_bytes(cfg), dtype=torch.uint8, device=logits.device)
    return _Router.apply(logits, cfg, mask, work)
