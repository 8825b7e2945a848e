"""Binding of the decoder-layer operators (include/loco_layer.h), and their differentiable forms.

The functions named loco_* have the name of the C entry point they call and only marshal arguments (in the native module
_layer_binding, csrc/layer_binding.cpp): every tensor, outputs included, is the caller's, nothing is allocated and nothing
synchronises.  `rotary`, `attention`, `router`, `norm`, `dispatch`, `combine` and `experts_product` wrap them as torch.autograd
functions that allocate their results, `experts_sort` and `clip_gradients` as plain ones.  All arithmetic runs in the CUDA kernels of
libloco_layer_b200.so; there is no CPU fallback: if the library cannot be loaded, the first call raises.
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
           "loco_router_backward", "loco_norm_forward", "loco_norm_backward", "loco_norm_backward_workspace_bytes",
           "loco_experts_sort", "loco_experts_sort_workspace_bytes", "loco_experts_clear", "loco_experts_clear_others", "loco_experts_dispatch", "loco_experts_combine",
           "loco_experts_combine_backward", "loco_experts_product", "loco_experts_product_weights", "loco_gradient_squares",
           "loco_gradient_squares_workspace_bytes", "loco_gradient_clip", "loco_layer_status", "loco_layer_launch_count")
FLAG_TIMEOUT = 1

# the C structures, packed in one go
_HEADS = struct.Struct("@Pqqq")                       # loco_heads_t
_TABLE = struct.Struct("@iiiffffff")                  # loco_rotary_table_t
_ROTARY = struct.Struct("@iiiiiiiii")                 # loco_rotary_t
_ATTENTION = struct.Struct("@iiiiiiiiiif4xPP")        # loco_attention_t
_ROUTER = struct.Struct("@iiiiff")                    # loco_router_t
_ROWS = struct.Struct("@Pq")                          # loco_rows_t
_NORM = struct.Struct("@iiiif")                       # loco_norm_t
_EXPERTS = struct.Struct("@iii4xqq")                  # loco_experts_t
_MATRICES = struct.Struct("@Pqq")                     # loco_matrices_t
_PRODUCT = struct.Struct("@i4xqiii4x")                # loco_product_t
_SPAN = struct.Struct("@PPQi4x")                      # loco_span_t

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
        L.loco_norm_forward.argtypes = [st, i64, st, st, vp, st, st, vp, vp]
        L.loco_norm_backward.argtypes = [st, i64, st, st, vp, st, st, vp, vp, u64, vp]
        L.loco_norm_backward_workspace_bytes.argtypes = [st]
        L.loco_experts_sort.argtypes = [i32, i64, i32, vp, vp, vp, vp, u64, vp]
        L.loco_experts_sort_workspace_bytes.argtypes = [i32]
        L.loco_experts_clear.argtypes = L.loco_experts_clear_others.argtypes = [i32, i32, i64, st, i32, vp, vp]
        L.loco_experts_dispatch.argtypes = [st, st, vp, st, vp]
        L.loco_experts_combine.argtypes = [st, st, vp, vp, st, vp]
        L.loco_experts_combine_backward.argtypes = [st, st, st, vp, vp, st, vp, vp]
        L.loco_experts_product.argtypes = [st, st, st, vp, st, vp]
        L.loco_experts_product_weights.argtypes = [st, st, st, vp, st, vp]
        L.loco_gradient_squares.argtypes = [st, i32, vp, vp, u64, vp]
        L.loco_gradient_squares_workspace_bytes.argtypes = []
        L.loco_gradient_clip.argtypes = [st, i32, vp, C.c_double, vp, vp]
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

    FLAG_TIMEOUT: a wait in an attention or product kernel ran out and that call's outputs are meaningless.  Nothing else reads the
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


# ---- norm ------------------------------------------------------------------------------------

def loco_norm_forward(x, y, weight=None, residual=None, total=None, scale=None, block: int = 0, eps: float = 1e-5, stream=None) -> None:
    """y = the root-mean-square norm of x + residual, times weight; total = x + residual as it is kept, in the type of x.

    x, residual, total, y: [rows, dim]; weight [dim].  y in float8_e4m3fn: with scale fp32 [rows, ceil(dim / block)], a scale
    for every 128 columns (block=128) or [rows, 1] (block=0); y * scale is the norm's output."""
    _check(_binding().norm_forward(x, y, weight, residual, total, scale, block, eps, _raw(stream)), "loco_norm_forward")


def loco_norm_backward_workspace_bytes(dim: int, dtype: torch.dtype = torch.bfloat16) -> int:
    """Bytes of loco_norm_backward's workspace for rows of `dim` elements."""
    return int(lib().loco_norm_backward_workspace_bytes(_NORM.pack(BF16 if dtype == torch.bfloat16 else 0, dim, 0, 0, 0.0)))


def loco_norm_backward(h, dy, dx, work=None, weight=None, dweight=None, dtotal=None, eps: float = 1e-5, stream=None) -> None:
    """Gradient of x (and of the residual alike) and of the weight, from h, what the norm was taken of (x + residual, or x).

    dtotal: the gradient that reaches h past the norm.  work: a CUDA tensor of loco_norm_backward_workspace_bytes() bytes,
    needed with dweight."""
    _check(_binding().norm_backward(h, dy, dx, work, weight, dweight, dtotal, eps, _raw(stream)), "loco_norm_backward")


# ---- experts ---------------------------------------------------------------------------------

def loco_experts_sort_workspace_bytes(experts: int) -> int:
    return int(lib().loco_experts_sort_workspace_bytes(experts))


def loco_experts_sort(index, offsets, place, work, stream=None) -> None:
    """Sort the router's choices index (int32 [tokens, top_k]) by expert, then token, then slot.

    offsets: int32 [experts + 1], the first row of every expert, then the number of rows; place: int32 [tokens, top_k], the
    row of a choice or -1; work: a CUDA tensor of loco_experts_sort_workspace_bytes() bytes."""
    _check(_binding().experts_sort(index, offsets, place, work, _raw(stream)), "loco_experts_sort")


def loco_experts_dispatch(x, place, rows, stream=None) -> None:
    """rows[place[t, j]] = x[t]; x [tokens, dim], rows [rows, dim].  Rows that no choice has are left as they are."""
    _check(_binding().experts_dispatch(x, place, rows, _raw(stream)), "loco_experts_dispatch")


def loco_experts_combine(rows, place, y, weight=None, stream=None) -> None:
    """y[t] = sum over j of weight[t, j] * rows[place[t, j]]; weight: fp32 [tokens, top_k], None for ones."""
    _check(_binding().experts_combine(rows, place, y, weight, _raw(stream)), "loco_experts_combine")


def loco_experts_combine_backward(dy, rows, place, weight, drows, dweight, stream=None) -> None:
    """drows[place[t, j]] = weight[t, j] * dy[t] and dweight[t, j] = dy[t] . rows[place[t, j]] (fp32)."""
    _check(_binding().experts_combine_backward(dy, rows, place, weight, drows, dweight, _raw(stream)), "loco_experts_combine_backward")


def loco_experts_clear(rows, offsets, stream=None) -> None:
    """Zeros in rows [rows, dim] from offsets[experts] on, which the other calls leave as they are."""
    _check(_binding().experts_clear(rows, offsets, _raw(stream)), "loco_experts_clear")


def loco_experts_clear_others(rows, offsets, stream=None) -> None:
    """Zeros in all rows of [rows, dim] that no expert has as loco_experts_product reads the offsets: ahead of offsets[0] too, and from
    the largest offset on."""
    _check(_binding().experts_clear_others(rows, offsets, _raw(stream)), "loco_experts_clear_others")


def loco_experts_product(x, w, offsets, y, transposed: bool = False, stream=None) -> None:
    """y[t] = x[t] @ w[e] for the rows t of every expert e, offsets[e] to offsets[e + 1]; bfloat16.

    x [rows, d_in], y [rows, d_out], w [experts, d_in, d_out], or [experts, d_out, d_in] and transposed.  The gradient of x is
    the same call on dy the other way round.  Rows outside every expert are left as they are."""
    _check(_binding().experts_product(x, w, offsets, y, transposed, _raw(stream)), "loco_experts_product")


def loco_experts_product_weights(a, b, offsets, dw, stream=None) -> None:
    """dw[e] = a[rows of e]^T @ b[rows of e], [experts, a's columns, b's columns]; zeros for an expert without rows."""
    _check(_binding().experts_product_weights(a, b, offsets, dw, _raw(stream)), "loco_experts_product_weights")


# ---- gradient --------------------------------------------------------------------------------

def loco_gradient_squares_workspace_bytes() -> int:
    return int(lib().loco_gradient_squares_workspace_bytes())


def loco_gradient_squares(gradients, squares, work, stream=None) -> None:
    """squares (fp64 [1]) = the sum of squares over a list of contiguous gradients (bfloat16 or fp32, of any shapes), within 6 * 2^-24.

    work: a CUDA tensor of loco_gradient_squares_workspace_bytes() bytes, zero before its first use."""
    _check(_binding().gradient_squares(gradients, squares, work, _raw(stream)), "loco_gradient_squares")


def loco_gradient_clip(gradients, outputs, squares, norm, max_norm: float, stream=None) -> None:
    """outputs = gradients times max_norm / sqrt(squares) where that is below one; norm (fp32 [1], or None) = sqrt(squares).

    An output may be its gradient itself; where nothing is to be scaled nothing is written to it then.  Autograd takes the outputs as
    changed, as after an operation of torch's in place."""
    _check(_binding().gradient_clip(gradients, outputs, squares, norm, max_norm, _raw(stream)), "loco_gradient_clip")


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


def _flat(t: torch.Tensor) -> torch.Tensor:
    """[rows, dim] of any leading dimensions, the rows contiguous; a copy where strides say so."""
    t = t.reshape(-1, t.shape[-1])
    return t if t.stride(1) == 1 or t.shape[1] == 1 else t.contiguous()


class _Norm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, weight, eps):
        flat, y = _flat(x), torch.empty(x.shape, dtype=x.dtype, device=x.device)
        total = None if residual is None else torch.empty(x.shape, dtype=x.dtype, device=x.device)
        loco_norm_forward(flat, _flat(y), weight=weight, residual=None if residual is None else _flat(residual),
                          total=None if total is None else _flat(total), eps=eps)
        ctx.save_for_backward(x if total is None else total, weight)
        ctx.eps, ctx.had_residual = eps, residual is not None
        ctx.set_materialize_grads(False)
        return y, total

    @staticmethod
    def backward(ctx, dy, dtotal):
        def compute(h, weight, dy, dtotal):
            if dy is None:
                return dtotal, None if weight is None else torch.zeros_like(weight)
            dx = torch.empty(h.shape, dtype=h.dtype, device=h.device)
            dweight = None if weight is None or not ctx.needs_input_grad[2] else torch.empty_like(weight, memory_format=torch.contiguous_format)
            work = None if dweight is None else torch.empty(loco_norm_backward_workspace_bytes(h.shape[-1], h.dtype), dtype=torch.uint8, device=h.device)
            loco_norm_backward(_flat(h), _flat(dy), _flat(dx), work, weight=weight, dweight=dweight, dtotal=None if dtotal is None else _flat(dtotal),
                               eps=ctx.eps)
            return dx, dweight
        if dy is None and dtotal is None:
            return None, None, None, None
        dx, dweight = _gradient("norm", compute, *ctx.saved_tensors, dy, dtotal)
        return dx, dx if ctx.had_residual else None, dweight, None


def norm(x, weight=None, residual=None, eps: float = 1e-5):
    """Root-mean-square norm of x [..., dim], times weight [dim]; with a residual (norm of x + residual, x + residual as it is kept).

    Differentiable once."""
    if residual is not None and residual.shape != x.shape and residual.numel() == x.numel() and residual.shape[-1] == x.shape[-1]:
        residual = residual.reshape(x.shape)         # other leading dimensions, which its gradient has to have again
    y, total = _Norm.apply(x, residual, weight, eps)
    return y if residual is None else (y, total)


def experts_sort(index, experts: int, work: Optional[torch.Tensor] = None):
    """(offsets, place) of the router's choices index [tokens, top_k], as loco_experts_sort.

    work: a workspace to keep between calls (loco_experts_sort_workspace_bytes() bytes); None allocates one."""
    offsets = torch.empty(experts + 1, dtype=torch.int32, device=index.device)
    place = torch.empty(index.shape, dtype=torch.int32, device=index.device)
    if work is None:
        work = torch.empty(loco_experts_sort_workspace_bytes(experts), dtype=torch.uint8, device=index.device)
    loco_experts_sort(index, offsets, place, work)
    return offsets, place


def _cleared(rows, offsets, others: bool = False):
    """`others`: where the offsets may be a caller's own.  Rows on the host are those of a stand-in for the kernels, whose offsets begin with 0."""
    (loco_experts_clear_others if others and rows.is_cuda else loco_experts_clear)(rows, offsets)
    return rows


class _Dispatch(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, place, offsets):
        rows = torch.empty(place.numel(), x.shape[1], dtype=x.dtype, device=x.device)
        loco_experts_dispatch(_flat(x), place, rows)
        ctx.save_for_backward(place)
        return _cleared(rows, offsets)

    @staticmethod
    def backward(ctx, drows):
        def compute(place, drows):
            dx = torch.empty(place.shape[0], drows.shape[1], dtype=drows.dtype, device=drows.device)
            loco_experts_combine(_flat(drows), place, dx)
            return dx
        return _gradient("dispatch", compute, *ctx.saved_tensors, drows), None, None


def dispatch(x, place, offsets):
    """The tokens x [tokens, dim] (or [..., dim]) in the order of experts_sort's (offsets, place): [tokens * top_k, dim], zeros in rows
    that no choice has.  Differentiable once."""
    return _Dispatch.apply(x.flatten(0, -2) if x.dim() > 2 else x, place, offsets)


class _Combine(torch.autograd.Function):
    @staticmethod
    def forward(ctx, rows, place, offsets, weight):
        y = torch.empty(place.shape[0], rows.shape[1], dtype=rows.dtype, device=rows.device)
        loco_experts_combine(_flat(rows), place, y, weight=weight)
        # without weights the gradient depends on nothing of the rows but their shape
        ctx.save_for_backward(None if weight is None else rows, place, offsets, weight)
        ctx.rows = rows.shape[0]
        return y

    @staticmethod
    def backward(ctx, dy):
        def compute(rows, place, offsets, weight, dy):
            drows = torch.empty(ctx.rows, dy.shape[1], dtype=dy.dtype, device=dy.device)
            if weight is None:
                loco_experts_dispatch(_flat(dy), place, drows)
                return _cleared(drows, offsets), None
            dweight = torch.empty(place.shape, dtype=torch.float32, device=dy.device)
            loco_experts_combine_backward(_flat(dy), _flat(rows), place, weight, drows, dweight)
            return _cleared(drows, offsets), dweight
        drows, dweight = _gradient("combine", compute, *ctx.saved_tensors, dy)
        return drows, None, None, dweight


def combine(rows, place, offsets, weight=None):
    """The experts' rows summed back to their tokens, with the choices' weights (fp32 [tokens, top_k]; None: ones).

    Differentiable once."""
    return _Combine.apply(rows.flatten(0, -2) if rows.dim() > 2 else rows, place, offsets, weight)


class _Product(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, offsets, transposed):
        y = torch.empty(x.shape[0], w.shape[1 if transposed else 2], dtype=x.dtype, device=x.device)
        loco_experts_product(x, w, offsets, y, transposed=transposed)
        ctx.save_for_backward(x, w, offsets)
        ctx.transposed = transposed
        return _cleared(y, offsets, others=True)

    @staticmethod
    def backward(ctx, dy):
        def compute(x, w, offsets, dy):
            dy = dy.contiguous()
            if dy.data_ptr() % 16:                   # a contiguous view, off the boundaries that the kernels need
                dy = dy.clone()
            dx = dw = None
            if ctx.needs_input_grad[0]:
                dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
                loco_experts_product(dy, w, offsets, dx, transposed=not ctx.transposed)
                _cleared(dx, offsets, others=True)
            if ctx.needs_input_grad[1]:
                dw = torch.empty(w.shape, dtype=w.dtype, device=w.device)
                loco_experts_product_weights(*((dy, x) if ctx.transposed else (x, dy)), offsets, dw)
            return dx, dw
        dx, dw = _gradient("experts_product", compute, *ctx.saved_tensors, dy)
        return dx, dw, None, None


def experts_product(x, w, offsets, transposed: bool = False):
    """x[t] @ w[e] for the rows t of every expert e, as loco_experts_product; zeros in rows that no expert has.

    Differentiable once."""
    return _Product.apply(x, w, offsets, transposed)


def clip_gradients(gradients, max_norm: float, work: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Scale a list of contiguous gradients down, in place, to a global norm of max_norm; returns the norm they had (fp32 [1]).

    No gradient may be there twice, or overlap another.  work: a workspace to keep between calls
    (loco_gradient_squares_workspace_bytes() bytes, zeroed once); None allocates one."""
    if not gradients:
        raise ValueError("clip_gradients: no gradients")
    device = gradients[0].device
    if work is None:
        work = torch.zeros(loco_gradient_squares_workspace_bytes(), dtype=torch.uint8, device=device)
    squares, norm = torch.empty(1, dtype=torch.float64, device=device), torch.empty(1, dtype=torch.float32, device=device)
    loco_gradient_squares(gradients, squares, work)
    loco_gradient_clip(gradients, gradients, squares, norm, max_norm)
    return norm
