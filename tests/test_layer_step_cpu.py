"""The example's parameters as views of its flat weights.  No GPU."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("d_ffn", [24, 20])
def test_views_are_the_flat_weights_in_the_order_of_the_parameters(d_ffn):
    """Of 20 columns each expert has its own: the products do not take them."""
    import decoder_layer_step as ex
    shape = ex.Shape(d_model=16, heads=2, heads_kv=1, head_dim=8, d_ffn=d_ffn, experts=3)
    sizes = shape.parameters()
    flat = torch.randn(sum(a * b for a, b in sizes.values())).requires_grad_()
    w = ex.views(shape, flat)
    assert ("w1" in w) == (d_ffn == 24)
    each = w if d_ffn == 20 else {n: w[n.split(".")[0]][int(n.split(".")[1])] if "." in n else w[n] for n in sizes}
    at = 0
    for name, (a, b) in sizes.items():
        part = flat.detach()[at:at + a * b]
        assert each[name].shape == (a, b) and torch.equal(each[name].detach().flatten(), part)
        assert each[name].data_ptr() == part.data_ptr(), "a copy"
        at += a * b
    aims = {n: torch.randn(s) for n, s in sizes.items()}
    grad, = torch.autograd.grad(sum((each[n] * aims[n]).sum() for n in sizes), flat)
    assert torch.equal(grad, torch.cat([aims[n].flatten() for n in sizes]))
