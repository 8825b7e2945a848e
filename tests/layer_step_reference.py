"""The example's decoder layer and its three losses in 64 bits, differentiated by torch.  `drop` leaves a term out of the
gradient, to see whether a comparison would notice."""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

# Every rounding to 16 bits moves a tensor by 2^-8 of its norm at most and by a third of that as a rule (half a unit, uniform).
# A gradient here passes a dozen to two dozen of them in a row, independent of each other: 1 to 2 times 2^-8 together.
# Three times that.
BOUND = 6 * 2.0 ** -8
TERMS = ("rotary", "shared head", "dq", "dk", "dv", "D", "weight normalisation", "weights", "softmax sum")


def inputs(shape, b, s, gen, device):
    """Weights, input and aim.  The input leans one way, so that the experts' counts differ."""
    w = {n: (torch.randn(size, generator=gen, device=device) * size[0] ** -0.5).to(torch.bfloat16) for n, size in shape.parameters().items()}
    lean = 0.7 * torch.randn(shape.d_model, generator=gen, device=device)
    x = (torch.randn(b, s, shape.d_model, generator=gen, device=device) + lean).to(torch.bfloat16)
    return w, x, torch.randn(x.shape, generator=gen, device=device)


def forward(shape, w, x, table, index, drop=()):
    """(output, balance, z) for the given choice of experts, coefficients of one; table [seq, head_dim] as the library's."""
    import decoder_layer_step as ex
    s, held = x.shape[1], lambda name, t: t.detach() if name in drop else t
    unit = lambda t: t * torch.rsqrt(t.square().mean(-1, keepdim=True) + 1e-5)
    qkv = (unit(x) @ w["qkv"]).unflatten(-1, (-1, shape.head_dim))
    q, k, v = qkv.split((shape.heads, shape.heads_kv, shape.heads_kv), 2)
    h = shape.head_dim // 2
    c, sn = table[:, None, :h], table[:, None, h:]

    def turn(t):
        y = torch.cat([t[..., :h] * c - t[..., h:] * sn, t[..., h:] * c + t[..., :h] * sn], -1)
        return y.detach() + t - t.detach() if "rotary" in drop else y
    q, k = held("dq", turn(q)), held("dk", turn(k))
    v = held("dv", v)
    k, v = (torch.stack([t] + [held("shared head", t)] * (shape.heads // shape.heads_kv - 1), 3).flatten(2, 3) for t in (k, v))
    a = torch.einsum("bihd,bjhd->bhij", q, k) / math.sqrt(shape.head_dim)
    a = a.masked_fill(~torch.ones(s, s, dtype=torch.bool, device=x.device).tril(), -math.inf)
    p = torch.exp(a - held("D", torch.logsumexp(a, -1, keepdim=True)))
    x = x + torch.einsum("bhij,bjhd->bihd", p, v).flatten(2) @ w["out"]
    rows = unit(x).flatten(0, 1)
    z = rows @ w["router"]
    p = torch.exp(z - held("softmax sum", torch.logsumexp(z, -1, keepdim=True)))
    weight = torch.gather(torch.softmax(z, -1), 1, index)
    weight = held("weights", weight / held("weight normalisation", weight.sum(1, keepdim=True)))
    n = torch.bincount(index.reshape(-1), minlength=shape.experts).to(z.dtype)
    balance = shape.experts * (n / index.numel() * p.mean(0)).sum()
    return x + ex.experts(shape, w, rows, index, weight).view_as(x), balance, torch.logsumexp(z, -1).square().mean()


def gradients(shape, w, x, aim, table, index, drop=()):
    """Per loss (output times aim, balance, z) the gradient of every parameter, qkv's by its three parts."""
    W = {n: t.detach().double().requires_grad_() for n, t in w.items()}
    y, balance, z = forward(shape, W, x.double(), table.double(), index, drop)
    out = []
    for loss in ((y * aim.double()).sum(), balance, z):
        grads = torch.autograd.grad(loss, list(W.values()), retain_graph=True, allow_unused=True)
        out.append(parts(shape, {n: torch.zeros_like(t) if g is None else g for (n, t), g in zip(W.items(), grads)}))
    return out


def parts(shape, grads):
    q, k, v = grads["qkv"].split([n * shape.head_dim for n in (shape.heads, shape.heads_kv, shape.heads_kv)], 1)
    return {"q": q, "k": k, "v": v, **{n: g for n, g in grads.items() if n != "qkv"}}


def far(got, want):
    """Names whose gradient is further off than BOUND of its norm."""
    return [n for n in want if float((got[n].double() - want[n]).norm()) > BOUND * float(want[n].norm())]
