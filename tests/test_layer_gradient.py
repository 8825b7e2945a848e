"""The gradient of the whole layer, parameter by parameter and loss by loss."""
import pytest
import torch

from tests import layer_step_reference as step


def small():
    import decoder_layer_step as ex
    return ex, ex.Shape(d_model=128, heads=4, heads_kv=2, head_dim=32, d_ffn=64)


@pytest.mark.parametrize("term", step.TERMS)
def test_the_comparison_notices_a_missing_term(term):
    """With the term left out of the 64-bit gradient itself, on the CPU."""
    _, shape = small()
    gen = torch.Generator()
    gen.manual_seed(5)
    w, x, aim = step.inputs(shape, 2, 90, gen, "cpu")
    angle = torch.arange(90.0, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(16, dtype=torch.float64) / 16)
    table = torch.cat([angle.cos(), angle.sin()], 1)
    index = torch.randint(0, 4, (180, 1), generator=gen)
    index = torch.cat([index, index + 1 + torch.randint(0, 4, (180, 1), generator=gen)], 1)
    want = step.gradients(shape, w, x, aim, table, index)
    assert not any(map(step.far, want, want))
    assert any(map(step.far, step.gradients(shape, w, x, aim, table, index, (term,)), want))


@pytest.mark.gpu
@pytest.mark.parametrize("seed", [5, 6])
def test_every_parameter_has_the_gradient_of_the_formulas(seed):
    from paper_2407_04480_b200 import layer
    ex, shape = small()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    b, s = 2, 150
    w, x, aim = step.inputs(shape, b, s, gen, "cuda")
    for t in w.values():
        t.requires_grad_()
    table = torch.empty(s, shape.head_dim, device="cuda")
    layer.loco_rotary_table(table)
    cfg = layer.Router(shape.experts, shape.top_k, balance_coef=1.0, z_coef=1.0)
    work = torch.zeros(layer.loco_router_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    y, counts, losses = ex.forward(shape, w, x, table, cfg, work)
    got = []
    for loss in ((y.float() * aim).sum(), losses[0], losses[1]):
        grads = torch.autograd.grad(loss, list(w.values()), retain_graph=True, allow_unused=True)
        got.append(step.parts(shape, {n: torch.zeros_like(t) if g is None else g for (n, t), g in zip(w.items(), grads)}))
    with torch.no_grad():                            # the choice, as the layer made it
        q, k, v = (ex.norm(x) @ w["qkv"]).unflatten(-1, (-1, shape.head_dim)).split((shape.heads, shape.heads_kv, shape.heads_kv), 2)
        o = layer.attention(*layer.rotary(q, k, table), v, causal=True)
        index = layer.router(ex.norm(x + o.flatten(2) @ w["out"]).flatten(0, 1) @ w["router"], cfg, work=work)[0].long()
    assert torch.equal(torch.bincount(index.flatten(), minlength=shape.experts).int(), counts[:shape.experts])
    want = step.gradients(shape, w, x, aim, table, index)
    for name, a, r in zip(("data", "balance", "z"), got, want):
        assert not step.far(a, r), (name, {n: float((a[n].double() - r[n]).norm() / r[n].norm()) for n in step.far(a, r)})
    assert layer.loco_layer_status() == 0
