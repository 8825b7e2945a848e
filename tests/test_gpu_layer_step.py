"""The decoder-layer operators together with the compressed gradient exchange: the example's training step."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_training_steps_learn():
    import decoder_layer_step as ex
    history = ex.run(steps=12, workers=2, batch=2, seq=160, report=lambda *_: None)
    assert all(h == h for h in history)
    assert history[-1] < 0.9 * history[0], history


def test_layer_gradient_matches_plain_torch():
    """Gradient of the whole layer against torch's differentiation of the same layer in 64 bits with the same choice.

    The layer rounds to 16 bits after every product, each rounding 2^-8 of its value; over its dozen products in a row the
    norm of the difference stays within 12 * 2^-8 of the gradient's."""
    import math

    import decoder_layer_step as ex
    from paper_2407_04480_b200 import layer
    shape = ex.Shape(d_model=128, heads=4, heads_kv=2, head_dim=32, d_ffn=64)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    b, s = 2, 150
    w = {n: (torch.randn(size, generator=g, device="cuda") * size[0] ** -0.5).to(torch.bfloat16).requires_grad_() for n, size in shape.parameters().items()}
    x = torch.randn(b, s, shape.d_model, generator=g, device="cuda").to(torch.bfloat16)
    table = torch.empty(s, shape.head_dim, device="cuda")
    layer.loco_rotary_table(table)
    cfg = layer.Router(shape.experts, shape.top_k, balance_coef=0.5, z_coef=0.1)
    work = torch.zeros(layer.loco_router_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    y, counts, losses = ex.forward(shape, w, x, table, cfg, work)
    aim = torch.randn(y.shape, generator=g, device="cuda")
    grads = torch.autograd.grad((y.float() * aim).mean() + losses.sum(), list(w.values()))

    # the same in 64 bits; the choice of experts is taken from logits rounded like the layer's
    W = {n: t.detach().double().requires_grad_() for n, t in w.items()}
    X = x.double()
    unit = lambda t: t * torch.rsqrt(t.square().mean(-1, keepdim=True) + 1e-5)
    qkv = (unit(X) @ W["qkv"]).unflatten(-1, (-1, shape.head_dim))
    q, k, v = qkv.split((shape.heads, shape.heads_kv, shape.heads_kv), 2)
    h = shape.head_dim // 2
    c, sn = table.double()[:, None, :h], table.double()[:, None, h:]
    turn = lambda t: torch.cat([t[..., :h] * c - t[..., h:] * sn, t[..., h:] * c + t[..., :h] * sn], -1)
    q, k = turn(q), turn(k).repeat_interleave(2, 2)
    v = v.repeat_interleave(2, 2)
    a = torch.einsum("bihd,bjhd->bhij", q, k) / math.sqrt(shape.head_dim)
    a = a.masked_fill(~torch.ones(s, s, dtype=torch.bool, device="cuda").tril(), -math.inf)
    o = torch.einsum("bhij,bjhd->bihd", torch.softmax(a, -1), v)
    Y = X + o.flatten(2) @ W["out"]
    H = unit(Y).flatten(0, 1)
    z = H @ W["router"]
    with torch.no_grad():
        wd = {n: t.detach() for n, t in w.items()}
        qk = (ex.norm(x) @ wd["qkv"]).unflatten(-1, (-1, shape.head_dim)).split((shape.heads, shape.heads_kv, shape.heads_kv), 2)
        rq, rk = layer.rotary(qk[0], qk[1], table)
        low = x + layer.attention(rq, rk, qk[2], causal=True).flatten(2) @ wd["out"]
        index = layer.router(ex.norm(low).flatten(0, 1) @ wd["router"], cfg, work=work)[0].long()
    p = torch.softmax(z, -1)
    weight = torch.gather(p, 1, index)
    weight = weight / weight.sum(1, keepdim=True)
    n = torch.bincount(index.reshape(-1), minlength=shape.experts).double()
    assert torch.equal(n.int(), counts[:shape.experts])
    Z = ex.experts(shape, W, H, index, weight)
    loss = ((Y + Z.view_as(Y)) * aim.double()).mean() + cfg.balance_coef * shape.experts * (n / (b * s * 2) * p.mean(0)).sum() \
        + cfg.z_coef * torch.logsumexp(z, -1).square().mean()
    want = torch.autograd.grad(loss, list(W.values()))
    got, ref = torch.cat([t.double().flatten() for t in grads]), torch.cat([t.flatten() for t in want])
    assert float((got - ref).norm()) <= 12 * 2.0 ** -8 * float(ref.norm())
