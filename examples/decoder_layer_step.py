"""Training steps of one Mixtral-shaped decoder layer with compressed gradients, on one GPU.

    python examples/decoder_layer_step.py [--steps 8] [--workers 2] [--full]

Every worker runs the layer on its own batch: rotary positions, causal attention with shared key heads, a top-2 router with
balance and z loss (paper_2407_04480_b200.layer), projections and experts as torch products.  Its gradient, flattened in
bfloat16 like a bucket of a trainer, goes through the send pass; the receive pass averages the workers' packed buffers and
applies the Adam-family step to the fp32 weights (paper_2407_04480_b200.loco).  The workers are simulated one after the other.
The data is random: a fixed target function of the input that the layer learns.
"""
from __future__ import annotations

import argparse
import os
import sys
from dataclasses import dataclass
from typing import Dict, List

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
    return (x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-5)).to(x.dtype)


def experts(shape: Shape, w: Dict[str, torch.Tensor], x: torch.Tensor, index: torch.Tensor, weight: torch.Tensor) -> torch.Tensor:
    y = torch.zeros_like(x)
    for e in range(shape.experts):
        token, place = torch.where(index == e)
        if token.numel():
            a, b = (x[token] @ w["w1.%d" % e]).chunk(2, -1)
            out = (torch.nn.functional.silu(a) * b) @ w["w2.%d" % e]
            y = y.index_add(0, token, out * weight[token, place, None].to(out.dtype))
    return y


def forward(shape: Shape, w: Dict[str, torch.Tensor], x: torch.Tensor, table: torch.Tensor, router: layer.Router, work: torch.Tensor):
    """(output, tokens per expert, balance and z loss) of x [batch, seq, d_model]."""
    b, s, _ = x.shape
    qkv = (norm(x) @ w["qkv"]).unflatten(-1, (-1, shape.head_dim))
    q, k, v = qkv.split((shape.heads, shape.heads_kv, shape.heads_kv), 2)
    q, k = layer.rotary(q, k, table)
    o = layer.attention(q, k, v, causal=True)
    x = x + o.flatten(2) @ w["out"]
    h = norm(x).flatten(0, 1)
    index, weight, counts, _, losses = layer.router(h @ w["router"], router, work=work)
    return x + experts(shape, w, h, index, weight).view_as(x), counts, losses


def run(shape: Shape = Shape(), steps: int = 8, workers: int = 2, batch: int = 2, seq: int = 320, seed: int = 0,
        lr: float = 2e-3, report=print) -> List[float]:
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
            parts, at = {}, 0
            for name, (a, b) in sizes.items():
                parts[name] = flat[at:at + a * b].view(a, b)
                at += a * b
            x = inputs[rank]
            y, counts, losses = forward(shape, parts, x, table, router, work)
            target = x + torch.tanh(x.cumsum(1) / (torch.arange(seq, device="cuda") + 1.0).sqrt()[:, None].to(x.dtype) @ turn)
            loss = (y.float() - target.float()).square().mean() + losses.sum()
            grad, = torch.autograd.grad(loss, flat)
            loco.loco_compensate_quantize_pack(states[rank], grad.contiguous(), comms[rank], k + 1)
            total += float(loss.detach()) / workers
            idle += int((counts[:shape.experts] == 0).sum())          # experts whose gradient segments are all zero
        loco.loco_unpack_dequant_reduce_adam(cfg, comms, n, *moments, theta, lr=lr, beta1=0.1, beta2=0.01, delta=1e-12)
        history.append(total)
        report("step %d: loss %.4f, idle experts over all workers %d" % (k, total, idle))
    if layer.loco_layer_status() & layer.FLAG_TIMEOUT:                # an attention kernel gave up: its outputs mean nothing
        raise RuntimeError("a wait of an attention kernel ran out: the steps' results are meaningless")
    return history


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=8)
    ap.add_argument("--workers", type=int, default=2)
    ap.add_argument("--full", action="store_true", help="Mixtral-8x7B's layer: 4096 wide, 32 / 8 heads, experts of 14336")
    a = ap.parse_args()
    run(MIXTRAL if a.full else Shape(), steps=a.steps, workers=a.workers)
