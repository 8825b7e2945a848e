"""Leading dimensions in the differentiable forms of the norm and the sorted experts, without a GPU: the kernels take rows, and a gradient
has the shape of what it is the gradient of."""
import pytest
import torch

from paper_2407_04480_b200 import layer
from tests.test_layer_experts_cpu import kernels, normal              # noqa: F401  (a fixture)


@pytest.mark.parametrize("x,residual", [((2, 3, 4), (6, 4)), ((6, 4), (1, 6, 4)), ((1, 4), (4,)), ((4,), (1, 1, 4)), ((3, 2, 4), (2, 3, 4))])
def test_a_residual_with_other_leading_dimensions_has_a_gradient_of_its_shape(kernels, x, residual):     # noqa: F811
    x, r = normal(*x).requires_grad_(), normal(*residual, seed=1).requires_grad_()
    y, total = layer.norm(x, residual=r)
    assert y.shape == total.shape == x.shape
    dx, dr = torch.autograd.grad([y, total], [x, r], [normal(*x.shape, seed=2), normal(*x.shape, seed=3)])
    assert dx.shape == x.shape and dr.shape == r.shape and torch.equal(dx.flatten(), dr.flatten())
    h = (x.detach().flatten() + r.detach().flatten()).view(x.shape).requires_grad_()
    want, = torch.autograd.grad([h * torch.rsqrt(h.square().mean(-1, keepdim=True) + 1e-5), h], h, [normal(*x.shape, seed=2), normal(*x.shape, seed=3)])
    assert torch.allclose(dx, want, atol=1e-12)


@pytest.mark.parametrize("shape", [(1, 4, 4), (2, 2, 4), (4, 1, 6), (2, 1, 2, 5)])
def test_tokens_with_leading_dimensions_are_laid_out_and_have_their_gradient(kernels, shape):            # noqa: F811
    place, offsets = torch.tensor([[2], [0], [-1], [1]], dtype=torch.int32), torch.tensor([0, 1, 3], dtype=torch.int32)
    x = normal(*shape).requires_grad_()
    flat = x.detach().reshape(4, -1)
    rows = layer.dispatch(x, place, offsets)
    assert torch.equal(rows.detach(), torch.stack([flat[1], flat[3], flat[0], torch.zeros_like(flat[0])]))
    dy = normal(*rows.shape, seed=4)
    dx, = torch.autograd.grad(rows, x, dy)
    assert dx.shape == x.shape and torch.equal(dx.reshape(4, -1), torch.stack([dy[2], dy[0], torch.zeros_like(dy[0]), dy[1]]))
    back = layer.combine(rows.detach().view(shape).requires_grad_(), place, offsets)
    assert torch.equal(back.detach()[[0, 1, 3]], flat[[0, 1, 3]]) and not back[2].any()


def test_clearing_the_rows_of_no_expert_refuses_what_clearing_those_behind_the_last_does():
    from paper_2407_04480_b200 import loco
    from tests.test_layer_experts_cpu import PTR, rows
    layer.lib()
    for call in (layer.lib().loco_experts_clear, layer.lib().loco_experts_clear_others):
        clear = lambda dtype=loco.BF16, d=64, n=4, r=rows(), e=8, o=PTR: call(dtype, d, n, r, e, o, None)
        for bad in (dict(dtype=2), dict(d=0), dict(n=-1), dict(r=None), dict(r=rows(stride=0)), dict(e=0), dict(e=513), dict(o=None)):
            assert clear(**bad) == loco.ERR_ARG, bad
        assert clear(o=PTR + 2) == loco.ERR_ALIGN and clear(r=rows(ptr=PTR + 1)) == loco.ERR_ALIGN and clear(n=0, r=rows(ptr=0)) == loco.OK
