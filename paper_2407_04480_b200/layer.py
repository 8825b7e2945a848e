"""Binding of the decoder-layer operators (include/loco_layer.h), and their differentiable forms.

The functions named loco_* have the name of the C entry point they call and only marshal arguments (in the native module
_layer_binding, csrc/layer_binding.cpp): every tensor, outputs included, is the caller's, nothing is allocated and nothing
synchronises.  `rotary`, `attention` and `router` wrap them as torch.autograd functions that allocate their results.  All
arithmetic runs in the CUDA kernels of libloco_layer_b200.so; there is no CPU fallback: if the library cannot be loaded, the
first call raises.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from dataclasses import dataclass
from typing import Optional

import torch

from .loco import BF16, LocoError, OK, status_string

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

# the C structures, packed in one go
_HEADS = struct.Struct("@Pqqq")                       # loco_heads_t
_TABLE = struct.Struct("@iiiffffff")                  # loco_rotary_table_t
_ROTARY = struct.Struct("@iiiiiiiii")                 # loco_rotary_t
_ATTENTION = struct.Struct("@iiiiiiiiiif4xPP")        # loco_attention_t
_ROUTER = struct.Struct("@iiiiff")                    # loco_router_t

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


_native = None


def _binding():
    """The native marshalling module; loads the library first, which it calls."""
    global _native
    if _native is None:
        lib()
        from . import _layer_binding
        _native = _layer_binding
    return _native


def _raw(stream: Optional[torch.cuda.Stream]) -> Optional[int]:
    """The raw stream for the native module; None lets it take the current one."""
    return None if stream is None else stream.cuda_stream


def loco_layer_launch_count() -> int:
    return int(lib().loco_layer_launch_count())


def loco_layer_status(stream=None) -> int:
    """Flags raised on the current device since the library was loaded; synchronises the stream.

    FLAG_TIMEOUT: a wait in an attention kernel ran out and that call's outputs are meaningless.  Nothing else reads the
    flag: a program asks where it synchronises anyway, once a step or a checkpoint."""
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
    if torch.cuda.current_device() != table.get_device():
        raise ValueError("the table lives on cuda:%d, which is not the current device" % table.get_device())
    cfg = _TABLE.pack(table.shape[1], table.shape[0], SCALINGS[scaling], base, factor, trained, slow, fast, magnitude)
    _check(lib().loco_rotary_table(cfg, table.data_ptr(), (torch.cuda.current_stream() if stream is None else stream).cuda_stream),
           "loco_rotary_table")


def loco_rotary_apply(table: torch.Tensor, q: torch.Tensor, k: Optional[torch.Tensor], q_out: torch.Tensor,
                      k_out: Optional[torch.Tensor], positions: Optional[torch.Tensor] = None, layout: str = "half",
                      inverse: bool = False, stream=None) -> None:
    """Rotate q [batch, seq, heads, dim] into q_out and k (or None) into k_out; an output may be its input.

    table: from loco_rotary_table; positions: int32 or int64 [batch, seq], None for 0, 1, 2, ... in every sample."""
    kind = LAYOUTS.get(layout)
    if kind is None:
        raise ValueError("layout must be one of %s" % (tuple(LAYOUTS),))
    _check(_binding().rotary_apply(table, q, k, q_out, k_out, positions, kind, inverse, _raw(stream)), "loco_rotary_apply")


# ---- attention -------------------------------------------------------------------------------

def loco_attention_forward(q, k, v, o, lse, causal: bool = False, scale: Optional[float] = None, len_q=None, len_k=None,
                           cu_q=None, cu_k=None, max_q: Optional[int] = None, max_k: Optional[int] = None, stream=None) -> None:
    """o = softmax(scale q k^T) v and the log-sum-exp of every row.

    Padded: q, o [batch, seq_q, heads, dim], k, v [batch, seq_k, heads_kv, dim], lse fp32 [batch, heads, seq_q], lengths
    len_q, len_k int32 [batch] (None: seq).  Packed: q, o [rows_q, heads, dim], k, v [rows_k, heads_kv, dim], lse
    [heads, rows_q], offsets cu_q, cu_k int32 [batch + 1] that ascend from 0 to rows_q and rows_k (rows outside every sample are
    not written), max_q, max_k the longest sample.  scale: None = 1/sqrt(dim)."""
    _check(_binding().attention_forward(q, k, v, o, lse, causal, scale, len_q, len_k, cu_q, cu_k, max_q, max_k, _raw(stream)),
           "loco_attention_forward")


def loco_attention_backward_workspace_bytes(q, k, cu_q=None, cu_k=None, max_q=None, max_k=None) -> int:
    """Bytes of loco_attention_backward's workspace for q and k of these shapes."""
    packed = cu_q is not None
    cfg = _ATTENTION.pack(cu_q.numel() - 1 if packed else q.shape[0], q.shape[-2], k.shape[-2], q.shape[-1], packed, q.shape[-3],
                          k.shape[-3], max_q if packed else 0, max_k if packed else 0, 0, 1.0, cu_q.data_ptr() if packed else 0,
                          cu_k.data_ptr() if packed else 0)
    return int(lib().loco_attention_backward_workspace_bytes(cfg))


def loco_attention_backward(q, k, v, o, lse, do, dq, dk, dv, work, causal: bool = False, scale: Optional[float] = None,
                            len_q=None, len_k=None, cu_q=None, cu_k=None, max_q: Optional[int] = None,
                            max_k: Optional[int] = None, stream=None) -> None:
    """dq, dk, dv from do and the forward pass's o and lse; arguments as loco_attention_forward.

    work: a contiguous CUDA tensor of loco_attention_backward_workspace_bytes() bytes or more."""
    _check(_binding().attention_backward(q, k, v, o, lse, do, dq, dk, dv, work, causal, scale, len_q, len_k, cu_q, cu_k, max_q,
                                         max_k, _raw(stream)), "loco_attention_backward")


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


def loco_router_forward(cfg: Router, logits, index, weight, counts, mean, losses, work, mask=None, stream=None) -> None:
    """Choice, weights, counts and losses of logits [tokens, experts]; see include/loco_layer.h for the outputs.

    mask: uint8 or bool [tokens]; work: a CUDA tensor of loco_router_workspace_bytes() bytes, zero before its first use."""
    _check(_binding().router_forward(cfg.experts, cfg.top_k, cfg.normalize, cfg.balance_coef, cfg.z_coef, logits, index, weight,
                                     counts, mean, losses, work, mask, _raw(stream)), "loco_router_forward")


def loco_router_backward(cfg: Router, logits, index, counts, dlogits, mask=None, dlosses=None, dweights=None,
                         stream=None) -> None:
    """Gradient of the logits from those of the two losses (fp32 [2]) and of the weights (fp32 [tokens, top_k])."""
    _check(_binding().router_backward(cfg.experts, cfg.top_k, cfg.normalize, cfg.balance_coef, cfg.z_coef, logits, index, counts,
                                      dlogits, mask, dlosses, dweights, _raw(stream)), "loco_router_backward")


# ---- differentiable forms --------------------------------------------------------------------

class _Gradient(torch.autograd.Function):
    """A backward pass as a node of its own, over everything that it depends on.  Its kernels write memory that autograd does
    not see into: what differentiates the gradient again has to pass here, and raises."""
    @staticmethod
    def forward(ctx, name, compute, *tensors):
        ctx.name = name
        return compute(*tensors)

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError("layer.%s can be differentiated once: its gradient has no gradient" % ctx.name)


def _gradient(name, compute, *tensors):
    """compute(*tensors), as a node only where a graph of the backward pass is wanted: a node costs some 10 us on the host."""
    return _Gradient.apply(name, compute, *tensors) if torch.is_grad_enabled() else compute(*tensors)


def _rotate(q, k, table, positions, layout, inverse):
    qo, ko = (None if t is None else torch.empty_like(t, memory_format=torch.contiguous_format) for t in (q, k))
    loco_rotary_apply(table, q, k, qo, ko, positions=positions, layout=layout, inverse=inverse)
    return qo, ko


class _Rotary(torch.autograd.Function):
    """Linear in q and k: the gradient is the transposed rotation, which is differentiable in turn."""
    @staticmethod
    def forward(ctx, q, k, table, positions, layout, inverse):
        ctx.save_for_backward(table, positions)
        ctx.how = (layout, inverse)
        return _rotate(q, k, table, positions, layout, inverse)

    @staticmethod
    def backward(ctx, dq, dk):
        table, positions = ctx.saved_tensors
        layout, inverse = ctx.how
        # contiguous: also a broadcast gradient gets memory of its own
        dq, dk = (None if t is None else t.contiguous() for t in (dq, dk))
        turn = _Rotary.apply if torch.is_grad_enabled() else _rotate
        return (*turn(dq, dk, table, positions, layout, not inverse), None, None, None, None)


def rotary(q, k, table, positions=None, layout: str = "half"):
    """Rotated queries and keys [batch, seq, heads, dim]; k may be None, and is then None in the result."""
    return _Rotary.apply(q, k, table, positions, layout, False)


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, causal, scale, lens, longest):
        o = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        lse = torch.empty((q.shape[1], q.shape[0]) if lens["cu_q"] is not None else (q.shape[0], q.shape[2], q.shape[1]),
                          dtype=torch.float32, device=q.device)
        loco_attention_forward(q, k, v, o, lse, causal=causal, scale=scale, **lens, **longest)
        ctx.save_for_backward(q, k, v, o, lse, *lens.values())
        ctx.how = (causal, scale, tuple(lens), longest)
        return o

    @staticmethod
    def backward(ctx, do):
        causal, scale, names, longest = ctx.how

        def compute(q, k, v, o, lse, *rest):
            lens, do = dict(zip(names, rest)), rest[-1].contiguous()
            if do.data_ptr() % 16:                   # a contiguous view, off the boundaries that the kernels need
                do = do.clone()
            dq, dk, dv = (torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k, v))
            work = torch.empty(loco_attention_backward_workspace_bytes(q, k, lens["cu_q"], lens["cu_k"], **longest), dtype=torch.uint8, device=q.device)
            loco_attention_backward(q, k, v, o, lse, do, dq, dk, dv, work, causal=causal, scale=scale, **lens, **longest)
            return dq, dk, dv
        return (*_gradient("attention", compute, *ctx.saved_tensors, do), None, None, None, None)


def attention(q, k, v, causal: bool = False, scale: Optional[float] = None, len_q=None, len_k=None, cu_q=None, cu_k=None,
              max_q: Optional[int] = None, max_k: Optional[int] = None):
    """softmax(scale q k^T) v; shapes and lengths as loco_attention_forward, on the current stream.  Differentiable once."""
    lens = dict(len_q=len_q, len_k=len_k, cu_q=cu_q, cu_k=cu_k)
    return _Attention.apply(q, k, v, causal, scale, lens, dict(max_q=max_q, max_k=max_k))


class _Router(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, cfg, mask, work):
        n, dev = logits.shape[0], logits.device
        index = torch.empty((n, cfg.top_k), dtype=torch.int32, device=dev)
        weight = torch.empty((n, cfg.top_k), dtype=torch.float32, device=dev)
        counts = torch.empty(cfg.experts + 1, dtype=torch.int32, device=dev)
        mean, losses = (torch.empty(size, dtype=torch.float32, device=dev) for size in (cfg.experts, 2))
        loco_router_forward(cfg, logits, index, weight, counts, mean, losses, work, mask=mask)
        ctx.save_for_backward(logits, index, counts, mask)
        ctx.cfg = cfg
        ctx.mark_non_differentiable(index, counts, mean)
        return index, weight, counts, mean, losses

    @staticmethod
    def backward(ctx, _index, dweight, _counts, _mean, dlosses):
        def compute(logits, index, counts, mask, dweight, dlosses):
            dlogits = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
            loco_router_backward(ctx.cfg, logits, index, counts, dlogits, mask=mask, dlosses=dlosses.contiguous(),
                                 dweights=dweight.contiguous())
            return dlogits
        return _gradient("router", compute, *ctx.saved_tensors, dweight, dlosses), None, None, None


def router(logits, cfg: Router, mask=None, work: Optional[torch.Tensor] = None):
    """(index, weight, counts, mean, losses) of logits [tokens, experts]; weight and losses are differentiable, once.

    work: a workspace to keep between calls (loco_router_workspace_bytes() bytes, zeroed once); None allocates one."""
    if work is None:
        work = torch.zeros(loco_router_workspace_bytes(cfg), dtype=torch.uint8, device=logits.device)
    return _Router.apply(logits, cfg, mask, work)
