"""Training steps of one Mixtral-shaped decoder layer with compressed gradients, on one GPU.

    python examples/decoder_layer_step.py [--steps 8] [--workers 2] [--clip 1.0] [--full]

Every worker runs the layer on its own batch: norms with the residual's addition, rotary positions, causal attention with shared
key heads, a top-2 router with balance and z loss, the tokens sorted by expert, the experts' products and the sum back
(paper_2407_04480_b200.layer), projections as torch products.  Its gradient, flattened in bfloat16 like a bucket of a trainer and
scaled down to a largest norm where one is given, goes through the send pass; the receive pass averages the workers' packed buffers and
applies the Adam-family step to the fp32 weights (paper_2407_04480_b200.loco).  The workers are simulated one after the other.
The data is random: a fixed target function of the input that the layer learns.
"""
from __future__ import annotations

import argparse
import os
import sys
from dataclasses import dataclass
from typing import Dict, List, Optional

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2407_04480_b200 import layer, loco  # noqa: E402


@dataclass(frozen=True)
class Shape:
    d_model: int = 256
    heads: int = 4
    heads_kv: int = 2
    head_dim: int = 64
    d_ffn: int = 512
    experts: int = 8
    top_k: int = 2

    def parameters(self) -> Dict[str, tuple]:
        p = {"qkv": (self.d_model, (self.heads + 2 * self.heads_kv) * self.head_dim),
             "out": (self.heads * self.head_dim, self.d_model), "router": (self.d_model, self.experts)}
        for e in range(self.experts):
            p["w1.%d" % e], p["w2.%d" % e] = (self.d_model, 2 * self.d_ffn), (self.d_ffn, self.d_model)
        return p


MIXTRAL = Shape(4096, 32, 8, 128, 14336, 8, 2)


def norm(x: torch.Tensor) -> torch.Tensor:
    """layer.norm's plain form."""
    return (x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-5)).to(x.dtype)


def products_take(shape: Shape) -> bool:
    """Whether the experts' widths and number are those that layer.experts_product takes; others go expert by expert."""
    return shape.d_model % 8 == 0 and shape.d_ffn % 8 == 0 and shape.experts <= 512


def sorted_experts(shape: Shape, w: Dict[str, torch.Tensor], x: torch.Tensor, index: torch.Tensor, weight: torch.Tensor) -> torch.Tensor:
    """experts() without a look at the counts on the host: the tokens sorted by expert, one product for all of them.  The matrices are
    w["w1"] and w["w2"], [experts, in, out] at any distance, or are put together of each expert's own."""
    offsets, place = layer.experts_sort(index, shape.experts)
    w1, w2 = (w[n] if n in w else torch.stack([w["%s.%d" % (n, e)] for e in range(shape.experts)]) for n in ("w1", "w2"))
    a, b = layer.experts_product(layer.dispatch(x, place, offsets), w1, offsets).chunk(2, -1)
    return layer.combine(layer.experts_product(torch.nn.functional.silu(a) * b, w2, offsets), place, offsets, weight)


def experts(shape: Shape, w: Dict[str, torch.Tensor], x: torch.Tensor, index: torch.Tensor, weight: torch.Tensor) -> torch.Tensor:
    y = torch.zeros_like(x)
    for e in range(shape.experts):
        token, place = torch.where(index == e)
        if token.numel():
            a, b = (x[token] @ w["w1.%d" % e]).chunk(2, -1)
            out = (torch.nn.functional.silu(a) * b) @ w["w2.%d" % e]
            y = y.index_add(0, token, out * weight[token, place, None].to(out.dtype))
    return y


def views(shape: Shape, flat: torch.Tensor) -> Dict[str, torch.Tensor]:
    """The parameters where they lie in the flat weights, the experts' matrices together.  Split, not sliced: the gradient of a split is
    put together once, that of every slice is as large as all weights."""
    sizes = shape.parameters()
    dense = [n for n in sizes if "." not in n]               # they come first
    parts = flat.split([sizes[n][0] * sizes[n][1] for n in dense] + [sum(a * b for n, (a, b) in sizes.items() if "." in n)])
    w = {n: t.view(sizes[n]) for n, t in zip(dense, parts)}
    (a1, b1), (a2, b2) = sizes["w1.0"], sizes["w2.0"]
    w1, w2 = parts[-1].view(shape.experts, a1 * b1 + a2 * b2).split((a1 * b1, a2 * b2), 1)
    w1, w2 = w1.unflatten(1, (a1, b1)), w2.unflatten(1, (a2, b2))
    if products_take(shape):
        return {**w, "w1": w1, "w2": w2}
    return {**w, **{"%s.%d" % (n, e): m[e] for n, m in (("w1", w1), ("w2", w2)) for e in range(shape.experts)}}


def forward(shape: Shape, w: Dict[str, torch.Tensor], x: torch.Tensor, table: torch.Tensor, router: layer.Router, work: torch.Tensor):
    """(output, tokens per expert, balance and z loss) of x [batch, seq, d_model]."""
    b, s, _ = x.shape
    qkv = (layer.norm(x) @ w["qkv"]).unflatten(-1, (-1, shape.head_dim))
    q, k, v = qkv.split((shape.heads, shape.heads_kv, shape.heads_kv), 2)
    q, k = layer.rotary(q, k, table)
    o = layer.attention(q, k, v, causal=True)
    h, x = layer.norm(o.flatten(2) @ w["out"], residual=x)
    h = h.flatten(0, 1)
    index, weight, counts, _, losses = layer.router(h @ w["router"], router, work=work)
    mixture = sorted_experts if products_take(shape) else experts
    return x + mixture(shape, w, h, index, weight).view_as(x), counts, losses


def run(shape: Shape = Shape(), steps: int = 8, workers: int = 2, batch: int = 2, seq: int = 320, seed: int = 0,
        lr: float = 2e-3, report=print, max_norm: Optional[float] = None) -> List[float]:
    """Training loss of every step."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    sizes = shape.parameters()
    n = sum(a * b for a, b in sizes.values())
    theta = torch.cat([torch.randn(a * b, generator=gen, device="cuda") * a ** -0.5 for a, b in sizes.values()])
    moments = [torch.zeros_like(theta) for _ in range(2)]
    cfg = loco.Config(bits=4, s=2.0 ** 12, s_e=2.0 ** 14, beta=0.5, reset_period=512, grad_dtype=loco.BF16, out_dtype=loco.BF16)
    states = [loco.State(cfg, n) for _ in range(workers)]
    comms = [torch.empty(loco.loco_packed_bytes(cfg, n), dtype=torch.uint8, device="cuda") for _ in range(workers)]
    table = torch.empty(seq, shape.head_dim, device="cuda")
    layer.loco_rotary_table(table)
    router = layer.Router(shape.experts, shape.top_k, balance_coef=0.02, z_coef=1e-3)
    work = torch.zeros(layer.loco_router_workspace_bytes(router), dtype=torch.uint8, device="cuda")
    inputs = [torch.randn(batch, seq, shape.d_model, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(workers)]
    turn = (torch.randn(shape.d_model, shape.d_model, generator=gen, device="cuda") * shape.d_model ** -0.5).to(torch.bfloat16)
    history = []
    for k in range(steps):
        total, idle = 0.0, 0
        for rank in range(workers):
            flat = theta.to(torch.bfloat16).requires_grad_()          # the weights every worker computes with
            x = inputs[rank]
            y, counts, losses = forward(shape, views(shape, flat), x, table, router, work)
            target = x + torch.tanh(x.cumsum(1) / (torch.arange(seq, device="cuda") + 1.0).sqrt()[:, None].to(x.dtype) @ turn)
            loss = (y.float() - target.float()).square().mean() + losses.sum()
            grad, = torch.autograd.grad(loss, flat)
            grad = grad.contiguous()
            if max_norm is not None:
                layer.clip_gradients([grad], max_norm)
            loco.loco_compensate_quantize_pack(states[rank], grad, comms[rank], k + 1)
            total += float(loss.detach()) / workers
            idle += int((counts[:shape.experts] == 0).sum())          # experts whose gradient segments are all zero
        loco.loco_unpack_dequant_reduce_adam(cfg, comms, n, *moments, theta, lr=lr, beta1=0.1, beta2=0.01, delta=1e-12)
        history.append(total)
        report("step %d: loss %.4f, idle experts over all workers %d" % (k, total, idle))
    if layer.loco_layer_status() & layer.FLAG_TIMEOUT:                # an attention or product kernel gave up: its outputs mean nothing
        raise RuntimeError("a wait of an attention or product kernel ran out: the steps' results are meaningless")
    return history


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=8)
    ap.add_argument("--workers", type=int, default=2)
    ap.add_argument("--full", action="store_true", help="Mixtral-8x7B's layer: 4096 wide, 32 / 8 heads, experts of 14336")
    ap.add_argument("--clip", type=float, default=None, help="largest norm of a worker's gradient")
    a = ap.parse_args()
    run(MIXTRAL if a.full else Shape(), steps=a.steps, workers=a.workers, max_norm=a.clip)
