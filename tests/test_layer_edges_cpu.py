"""Host-side edges of the decoder-layer operators that need no GPU: sizes past every limit, and what the differentiable forms
hand to the kernels, which stand-ins in plain torch take the place of."""
import struct

import pytest
import torch

from paper_2407_04480_b200 import build as loco_build
from paper_2407_04480_b200 import layer, loco

PTR = 1 << 20                    # 16-byte aligned, never read


@pytest.fixture(scope="module", autouse=True)
def built():
    loco_build.build()


@pytest.mark.parametrize("tokens", [(1 << 31) // 4, 1 << 61, 1 << 62, (1 << 63) - 1])
def test_router_refuses_token_counts_whose_product_with_top_k_overflows(tokens):
    cfg = layer.Router(8, 4).c()
    L = layer.lib()
    assert L.loco_router_forward(cfg, tokens, PTR, 8, None, PTR, PTR, PTR, PTR, PTR, PTR, 1 << 30, None) == loco.ERR_ARG
    assert L.loco_router_backward(cfg, tokens, PTR, 8, None, PTR, PTR, None, None, PTR, 8, None) == loco.ERR_ARG


def heads(batch=0, row=0, head=0):
    return struct.pack("@Pqqq", PTR, batch, row, head)


def attention_cfg(batch=1, hq=1, hk=1, sq=1, sk=1):
    return layer._ATTENTION.pack(batch, hq, hk, 64, 0, sq, sk, 0, 0, 0, 0.125, 0, 0)


@pytest.mark.parametrize("size", [dict(batch=1 << 16, hq=512, hk=512, sk=65 * 128), dict(batch=1 << 16, hq=512, hk=512, sq=65 * 128),
                                  dict(batch=1 << 16, hq=512, hk=512, sq=129 * 128),
                                  dict(batch=1 << 30, hq=1 << 30, hk=1 << 30, sq=1 << 12, sk=1 << 12),
                                  dict(batch=1 << 16, hq=1 << 16, hk=1)])
def test_attention_refuses_more_blocks_than_a_launch_holds_before_it_launches_any(size):
    """More than 2^31 blocks in one of the call's kernels alone, or more than 64 bits hold."""
    cfg, x, L = attention_cfg(**size), heads(8, 8, 8), layer.lib()
    before = layer.loco_layer_launch_count()
    # the workspace is a number here, large enough for any of these
    assert L.loco_attention_backward(cfg, x, x, x, x, PTR, x, x, x, x, PTR, (1 << 64) - 1, None) == loco.ERR_UNSUPPORTED
    tiles = -(-size.get("sq", 1) // 256)                 # the forward kernel's, of 256 queries
    if tiles * size["batch"] * size["hq"] >= 1 << 31:
        assert L.loco_attention_forward(cfg, x, x, x, x, PTR, None) == loco.ERR_UNSUPPORTED
    assert layer.loco_layer_launch_count() == before


@pytest.mark.parametrize("zero", ["batch", "row", "head"])
def test_outputs_that_repeat_memory_are_refused(zero):
    """Inputs may (expanded tensors); of an output several threads would write the same place."""
    L, good = layer.lib(), dict(batch=2048, row=256, head=64)
    x, bad = heads(*good.values()), heads(*{**good, zero: 0}.values())
    cfg = attention_cfg(batch=2, hq=4, hk=4, sq=8, sk=8)
    size = L.loco_attention_backward_workspace_bytes(cfg)
    assert L.loco_attention_forward(cfg, x, x, x, bad, PTR, None) == loco.ERR_ARG
    for outs in ((bad, x, x), (x, bad, x), (x, x, bad)):
        assert L.loco_attention_backward(cfg, x, x, x, x, PTR, x, *outs, PTR, size, None) == loco.ERR_ARG
    cfg = layer._ROTARY.pack(loco.BF16, 0, 64, 64, 2, 8, 8, 0, 0)
    assert L.loco_rotary_apply(cfg, PTR, None, x, bad, struct.pack("@i", 4), 1, None) == loco.ERR_ARG
    assert L.loco_router_backward(layer.Router(8, 2).c(), 4, PTR, 8, None, PTR, PTR, None, None, PTR, 0, None) == loco.ERR_ARG


def test_a_binding_of_another_torch_is_out_of_date(monkeypatch):
    """It needs that torch's libraries; the sources alone would not show it."""
    import importlib.metadata as metadata
    assert not loco_build.stale_binding()
    real = metadata.version
    monkeypatch.setattr(metadata, "version", lambda name: "99.0" if name == "torch" else real(name))
    assert loco_build.stale_binding()


# ---- differentiable forms, with plain torch in the place of the kernels

@pytest.fixture
def kernels(monkeypatch):
    """Stand-ins that fill the outputs as the kernels do, out of autograd's sight; calls are noted as (name, arguments)."""
    calls = []

    def stand_in(name):
        def place(fn):
            def call(*a, **kw):
                calls.append((name, a, kw))
                with torch.no_grad():
                    fn(*a, **kw)
            monkeypatch.setattr(layer, name, call)
            return fn
        return place

    @stand_in("loco_rotary_apply")
    def _(table, q, k, qo, ko, positions=None, layout="half", inverse=False):
        for x, y in ((q, qo), (k, ko)):
            if x is not None:
                y.copy_(x * 2)                   # its own transpose

    @stand_in("loco_attention_forward")
    def _(q, k, v, o, lse, **kw):
        o.copy_(q * 3)
        lse.zero_()

    @stand_in("loco_attention_backward")
    def _(q, k, v, o, lse, do, dq, dk, dv, work, **kw):
        dq.copy_(do * 3)
        dk.zero_()
        dv.zero_()

    @stand_in("loco_router_forward")
    def _(cfg, logits, index, weight, counts, mean, losses, work, mask=None):
        weight.copy_(logits[:, :cfg.top_k])
        for t in (index, counts, mean, losses):
            t.zero_()

    @stand_in("loco_router_backward")
    def _(cfg, logits, index, counts, dlogits, mask=None, dlosses=None, dweights=None):
        dlogits.zero_()
        dlogits[:, :cfg.top_k] = dweights
    return calls


def forms():
    """(operands that require a gradient, a differentiable output) of each form."""
    heads = [torch.randn(1, 4, 2, 8, requires_grad=True) for _ in range(3)]
    z = torch.randn(5, 8, requires_grad=True)
    return {"rotary": (heads[0], lambda: layer.rotary(heads[0], heads[1], torch.zeros(4, 8))[0]),
            "attention": (heads[0], lambda: layer.attention(*heads)),
            "router": (z, lambda: layer.router(z, layer.Router(8, 2), work=torch.zeros(1))[1])}


@pytest.mark.parametrize("form", ["attention", "router"])
def test_a_second_derivative_is_refused(kernels, form):
    """The gradient of a gradient would lose the terms that go through the backward kernel."""
    x, value = forms()[form]
    for loss in (lambda: (value() ** 3).sum(), lambda: (value() ** 3).sum() + (x ** 3).sum()):
        grad, = torch.autograd.grad(loss(), x, create_graph=True)
        assert torch.isfinite(grad).all()
        with pytest.raises(RuntimeError, match="differentiated once"):
            torch.autograd.grad((grad ** 2).sum(), x)
        with pytest.raises(RuntimeError, match="differentiated once"):
            torch.autograd.grad(loss(), x, create_graph=True)[0].square().sum().backward()
        # the first one stays as it is, and frees its graph
        torch.autograd.grad(loss(), x)[0].square().sum()


def test_rotary_has_every_derivative(kernels):
    """Its gradient is a rotation again; the stand-in is a product with 2."""
    x, value = forms()["rotary"]

    def second(y):
        grad, = torch.autograd.grad((y() ** 3 + x ** 3).sum(), x, create_graph=True)
        return grad, torch.autograd.grad((grad ** 2).sum(), x)[0]
    for got, want in zip(second(value), second(lambda: 2 * x)):
        assert torch.allclose(got, want)
    assert [c[2]["inverse"] for c in kernels] == [False, True, False, True]


def lengths(packed):
    if packed:
        cu = torch.tensor([0, 3, 4], dtype=torch.int32)
        return (4, 2, 8), dict(cu_q=cu, cu_k=cu.clone(), max_q=3, max_k=3)
    return (2, 4, 2, 8), dict(len_q=torch.tensor([4, 2], dtype=torch.int32), len_k=torch.tensor([1, 4], dtype=torch.int32))


@pytest.mark.parametrize("changed", ["len_q", "len_k", "cu_q", "cu_k"])
def test_attention_notices_lengths_that_change_before_the_backward_pass(kernels, changed):
    shape, lens = lengths(changed.startswith("cu"))
    q, k, v = (torch.randn(shape, requires_grad=True) for _ in range(3))
    o = layer.attention(q, k, v, causal=True, **lens)
    lens[changed] += 1
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        o.sum().backward()


@pytest.mark.parametrize("packed", [False, True])
def test_attention_hands_the_same_lengths_to_both_passes(kernels, packed):
    shape, lens = lengths(packed)
    q, k, v = (torch.randn(shape, requires_grad=True) for _ in range(3))
    layer.attention(q, k, v, causal=True, scale=0.3, **lens).sum().backward()
    (_, _, there), (_, _, back) = kernels
    assert there.keys() == back.keys() and there["causal"] is True and there["scale"] == 0.3
    for name, value in lens.items():
        assert there[name] is value and (back[name] == value if isinstance(value, int) else torch.equal(back[name], value))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float64])
def test_router_results_do_not_take_the_default_type(kernels, dtype):
    was = torch.get_default_dtype()
    torch.set_default_dtype(dtype)
    try:
        layer.router(torch.randn(5, 8, dtype=torch.float32), layer.Router(8, 2), work=torch.zeros(1))
    finally:
        torch.set_default_dtype(was)
    (_, (_, _, index, weight, counts, mean, losses, _), _), = kernels
    assert [t.dtype for t in (index, weight, counts, mean, losses)] == [torch.int32, torch.float32, torch.int32, torch.float32, torch.float32]


def test_attention_takes_a_gradient_that_is_a_view_off_every_boundary(kernels):
    """torch.cat hands on a contiguous view at an odd offset; the kernels need 16-byte boundaries."""
    q, k, v = (torch.randn(1, 4, 2, 8, dtype=torch.bfloat16).requires_grad_() for _ in range(3))
    o = layer.attention(q, k, v)
    joined = torch.cat([torch.zeros(3, dtype=torch.bfloat16), o.flatten()])
    w = torch.randn(joined.shape).to(torch.bfloat16)
    got, = torch.autograd.grad(joined, q, w)
    _, args, _ = kernels[-1]
    assert args[5].is_contiguous() and args[5].data_ptr() % 16 == 0
    assert torch.equal(got, w[3:].view_as(q) * 3)


@pytest.mark.parametrize("name", ["stream", "len", "out"])
def test_differentiable_attention_takes_no_other_argument(kernels, name):
    """Its results belong to the current stream: work sent to another one would outlive them."""
    q, k, v = (torch.randn(1, 4, 2, 8) for _ in range(3))
    with pytest.raises(TypeError):
        layer.attention(q, k, v, **{name: None})
    assert not kernels


def test_rotary_takes_queries_alone(kernels):
    q = torch.randn(1, 4, 2, 8, requires_grad=True)
    y, none = layer.rotary(q, None, torch.zeros(4, 8))
    assert none is None and torch.equal(y, 2 * q)
    grad, = torch.autograd.grad(y, q, torch.ones_like(y))
    assert torch.equal(grad, torch.full_like(q, 2.0)) and [c[1][2] for c in kernels] == [None, None]
