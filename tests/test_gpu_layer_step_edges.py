"""The example's layer with its experts' matrices where they lie in the flat weights."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_matrices_in_the_flat_weights_give_the_results_of_their_copies():
    import decoder_layer_step as ex
    from paper_2407_04480_b200 import layer
    shape = ex.Shape(d_model=128, heads=4, heads_kv=2, head_dim=32, d_ffn=64)
    g = torch.Generator(device="cuda")
    g.manual_seed(8)
    sizes = shape.parameters()
    flat = torch.cat([torch.randn(a * b, generator=g, device="cuda") * a ** -0.5 for a, b in sizes.values()]).to(torch.bfloat16).requires_grad_()
    x = torch.randn(2, 150, shape.d_model, generator=g, device="cuda").to(torch.bfloat16)
    table = torch.empty(150, shape.head_dim, device="cuda")
    layer.loco_rotary_table(table)
    cfg = layer.Router(shape.experts, shape.top_k, balance_coef=0.5, z_coef=0.1)
    work = torch.zeros(layer.loco_router_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    copies = dict(zip(sizes, (t.view(s) for t, s in zip(flat.split([a * b for a, b in sizes.values()]), sizes.values()))))
    results = []
    for w in (ex.views(shape, flat), copies):
        y, counts, losses = ex.forward(shape, w, x, table, cfg, work)
        grad, = torch.autograd.grad(y.float().square().mean() + losses.sum(), flat)
        results.append((y.detach(), counts, losses.detach(), grad))
    assert all(torch.equal(a, b) for a, b in zip(*results))


@pytest.mark.parametrize("change", [dict(d_ffn=100), dict(d_model=132)])
def test_widths_that_the_products_do_not_take_go_expert_by_expert(change):
    """The step runs, with a gradient for every weight that is used."""
    import decoder_layer_step as ex
    from paper_2407_04480_b200 import layer
    shape = ex.Shape(**{**dict(d_model=128, heads=4, heads_kv=2, head_dim=32, d_ffn=64), **change})
    assert not ex.products_take(shape)
    history = ex.run(shape, steps=2, workers=1, batch=1, seq=70, report=lambda *_: None)
    assert all(h == h for h in history)
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    sizes = shape.parameters()
    flat = torch.cat([torch.randn(a * b, generator=g, device="cuda") * a ** -0.5 for a, b in sizes.values()]).to(torch.bfloat16).requires_grad_()
    x = torch.randn(1, 70, shape.d_model, generator=g, device="cuda").to(torch.bfloat16)
    table = torch.empty(70, shape.head_dim, device="cuda")
    layer.loco_rotary_table(table)
    cfg = layer.Router(shape.experts, shape.top_k)
    work = torch.zeros(layer.loco_router_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    y, _, losses = ex.forward(shape, ex.views(shape, flat), x, table, cfg, work)
    grad, = torch.autograd.grad(y.float().square().mean() + losses.sum(), flat)
    assert torch.isfinite(grad).all() and bool(grad.any())
