"""Host-side checks of the decoder-layer operators that need no GPU: exported symbols, structure layouts, refusals.

A refusal is returned before anything touches a device, so the addresses in these calls are never used."""
import ctypes as C
import os
import re
import struct

import pytest

from paper_2407_04480_b200 import build as loco_build
from paper_2407_04480_b200 import layer, loco

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PTR = 1 << 20                    # 16-byte aligned, never read


@pytest.fixture(scope="module", autouse=True)
def built():
    loco_build.build()


def test_library_exports_every_declared_symbol():
    text = open(os.path.join(ROOT, "include", "loco_layer.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = sorted(set(re.findall(r"\b(loco_[a-z0-9_]+)\s*\(", text)))
    assert sorted(layer.EXPORTS) == names
    L = C.CDLL(layer.LIB_PATH)
    for name in names:
        assert hasattr(L, name) and hasattr(layer, name), name


def test_packed_structures_have_the_sizes_of_the_c_ones():
    class heads(C.Structure):
        _fields_ = [("ptr", C.c_void_p), ("b", C.c_int64), ("r", C.c_int64), ("h", C.c_int64)]

    class attention(C.Structure):
        _fields_ = [(n, C.c_int32) for n in ("batch", "hq", "hk", "d", "packed", "sq", "sk", "mq", "mk", "causal")] + [
            ("scale", C.c_float), ("lq", C.c_void_p), ("lk", C.c_void_p)]

    class router(C.Structure):
        _fields_ = [(n, C.c_int32) for n in ("dtype", "experts", "k", "norm")] + [("a", C.c_float), ("b", C.c_float)]

    class table(C.Structure):
        _fields_ = [(n, C.c_int32) for n in ("r", "positions", "scaling")] + [
            (n, C.c_float) for n in ("base", "factor", "trained", "slow", "fast", "magnitude")]
    assert layer._HEADS.size == C.sizeof(heads)
    assert layer._ATTENTION.size == C.sizeof(attention)
    assert layer._ROUTER.size == C.sizeof(router)
    assert layer._TABLE.size == C.sizeof(table)
    assert layer._ROTARY.size == 9 * 4
    a = attention.from_buffer_copy(layer._ATTENTION.pack(1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 0.5, 11, 12))
    assert [getattr(a, n) for n, _ in attention._fields_] == [1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 0.5, 11, 12]


def heads(ptr=PTR, b=0, r=128, h=128):
    return struct.pack("@Pqqq", ptr, b, r, h)


def attention_cfg(batch=1, hq=4, hk=2, d=64, packed=0, sq=16, sk=16, mq=0, mk=0, causal=0, scale=0.125, lq=0, lk=0):
    return layer._ATTENTION.pack(batch, hq, hk, d, packed, sq, sk, mq, mk, causal, scale, lq, lk)


def forward(cfg, q=None, k=None, v=None, o=None, lse=PTR):
    x = heads()
    return layer.lib().loco_attention_forward(cfg, q or x, k or x, v or x, o or x, lse, None)


@pytest.mark.parametrize("bad,code", [
    (dict(hk=3), loco.ERR_ARG), (dict(hk=0), loco.ERR_ARG), (dict(hq=0), loco.ERR_ARG), (dict(batch=-1), loco.ERR_ARG),
    (dict(d=0), loco.ERR_ARG), (dict(d=136), loco.ERR_UNSUPPORTED), (dict(d=60), loco.ERR_UNSUPPORTED), (dict(sq=-1), loco.ERR_ARG),
    (dict(scale=float("nan")), loco.ERR_ARG), (dict(scale=float("inf")), loco.ERR_ARG), (dict(packed=1), loco.ERR_ARG),
    (dict(packed=1, lq=PTR, lk=PTR, mq=17), loco.ERR_ARG), (dict(lq=PTR + 2), loco.ERR_ALIGN)])
def test_attention_refuses_a_bad_configuration(bad, code):
    assert forward(attention_cfg(**bad)) == code
    assert layer.lib().loco_attention_backward_workspace_bytes(attention_cfg(**bad)) == 0


def test_attention_refuses_bad_operands():
    cfg = attention_cfg()
    L = layer.lib()
    assert forward(None) == loco.ERR_ARG
    assert L.loco_attention_forward(cfg, None, heads(), heads(), heads(), PTR, None) == loco.ERR_ARG
    assert forward(cfg, q=heads(ptr=0)) == loco.ERR_ARG
    assert forward(cfg, v=heads(r=-128)) == loco.ERR_ARG
    assert forward(cfg, k=heads(ptr=PTR + 8)) == loco.ERR_ALIGN
    assert forward(cfg, k=heads(h=124)) == loco.ERR_ALIGN
    assert forward(attention_cfg(batch=2), o=heads(b=4)) == loco.ERR_ALIGN
    assert forward(cfg, lse=None) == loco.ERR_ARG
    assert forward(cfg, lse=PTR + 2) == loco.ERR_ALIGN
    need = L.loco_attention_backward_workspace_bytes(cfg)
    assert need >= 4 * 4 * 16
    x = heads()
    assert L.loco_attention_backward(cfg, x, x, x, x, PTR, x, x, x, x, PTR, need - 1, None) == loco.ERR_SIZE
    assert L.loco_attention_backward(cfg, x, x, x, x, PTR, x, x, x, x, None, need, None) == loco.ERR_ARG
    assert L.loco_attention_backward(cfg, x, x, x, x, PTR, x, x, x, heads(ptr=0), PTR, need, None) == loco.ERR_ARG
    assert L.loco_attention_backward(cfg, x, x, x, x, PTR, x, x, x, x, PTR + 8, need, None) == loco.ERR_ALIGN
    # nothing to do
    assert forward(attention_cfg(batch=0), q=heads(ptr=0)) == loco.OK
    assert forward(attention_cfg(sq=0), q=heads(ptr=0), o=heads(ptr=0)) == loco.OK


def rotary_cfg(dtype=loco.BF16, layout=0, d=64, r=64, batch=1, seq=4, positions=8, pb=0, inverse=0):
    return layer._ROTARY.pack(dtype, layout, d, r, batch, seq, positions, pb, inverse)


def rotate(cfg, x=None, y=None, n=(4, 0), count=1, table=PTR, at=None):
    x = x or heads() + heads()
    return layer.lib().loco_rotary_apply(cfg, table, at, x, y or x, struct.pack("@ii", *n), count, None)


@pytest.mark.parametrize("bad", [dict(dtype=2), dict(layout=2), dict(d=0), dict(r=0), dict(r=63), dict(r=66), dict(d=2048, r=2),
                                 dict(batch=-1), dict(seq=-1), dict(seq=9), dict(positions=0), dict(batch=1 << 16, seq=1 << 15, positions=1 << 15)])
def test_rotary_refuses_a_bad_configuration(bad):
    assert rotate(rotary_cfg(**bad)) == loco.ERR_ARG


def test_rotary_refuses_bad_operands():
    ok = rotary_cfg()
    assert rotate(None) == loco.ERR_ARG
    assert rotate(ok, count=0) == loco.ERR_ARG and rotate(ok, count=3) == loco.ERR_ARG
    assert rotate(ok, n=(-1, 0)) == loco.ERR_ARG
    assert rotate(ok, x=heads(ptr=0)) == loco.ERR_ARG
    assert rotate(ok, x=heads(ptr=PTR + 1)) == loco.ERR_ALIGN
    assert rotate(ok, table=None) == loco.ERR_ARG and rotate(ok, table=PTR + 4) == loco.ERR_ALIGN
    assert rotate(rotary_cfg(pb=3), at=PTR) == loco.ERR_ARG
    assert rotate(rotary_cfg(pb=8), at=PTR + 4) == loco.ERR_ALIGN
    assert rotate(rotary_cfg(batch=0)) == loco.OK and rotate(ok, n=(0, 0)) == loco.OK


def table(r=64, positions=8, scaling=0, base=1e4, factor=1.0, trained=4096.0, slow=1.0, fast=32.0, magnitude=1.0):
    return layer._TABLE.pack(r, positions, scaling, base, factor, trained, slow, fast, magnitude)


@pytest.mark.parametrize("bad", [dict(r=0), dict(r=7), dict(r=1026), dict(positions=0), dict(scaling=3), dict(base=0.0), dict(base=float("inf")),
                                 dict(scaling=1, factor=0.0), dict(scaling=2, trained=0.0), dict(scaling=2, slow=-1.0),
                                 dict(scaling=2, slow=5.0, fast=5.0), dict(magnitude=float("nan"))])
def test_rotary_table_refuses_a_bad_configuration(bad):
    assert layer.lib().loco_rotary_table(table(**bad), PTR, None) == loco.ERR_ARG


def test_rotary_table_refuses_bad_operands():
    assert layer.lib().loco_rotary_table(None, PTR, None) == loco.ERR_ARG
    assert layer.lib().loco_rotary_table(table(), None, None) == loco.ERR_ARG
    assert layer.lib().loco_rotary_table(table(), PTR + 4, None) == loco.ERR_ALIGN


def route(cfg, tokens=4, logits=PTR, stride=8, index=PTR, weight=PTR, counts=PTR, mean=PTR, losses=PTR, work=PTR, size=1 << 30):
    return layer.lib().loco_router_forward(cfg, tokens, logits, stride, None, index, weight, counts, mean, losses, work, size, None)


@pytest.mark.parametrize("bad", [dict(dtype=2), dict(experts=0), dict(experts=513), dict(k=0), dict(k=9), dict(experts=64, k=17),
                                 dict(a=float("nan")), dict(z=float("inf"))])
def test_router_refuses_a_bad_configuration(bad):
    c = dict(dtype=loco.BF16, experts=8, k=2, norm=1, a=0.01, z=0.0)
    c.update(bad)
    cfg = layer._ROUTER.pack(*c.values())
    assert route(cfg) == loco.ERR_ARG
    assert layer.lib().loco_router_workspace_bytes(cfg) == 0
    assert layer.lib().loco_router_backward(cfg, 4, PTR, 8, None, PTR, PTR, None, None, PTR, 8, None) == loco.ERR_ARG


def test_router_refuses_bad_operands():
    cfg = layer.Router(8, 2).c()
    assert route(None) == loco.ERR_ARG
    assert route(cfg, tokens=-1) == loco.ERR_ARG and route(cfg, tokens=1 << 30) == loco.ERR_ARG
    for name in ("logits", "index", "weight", "counts", "mean", "losses", "work"):
        assert route(cfg, **{name: None}) == loco.ERR_ARG, name
        assert route(cfg, **{name: PTR + 1}) == loco.ERR_ALIGN, name
    assert route(cfg, size=layer.lib().loco_router_workspace_bytes(cfg) - 1) == loco.ERR_SIZE
    back = lambda **a: layer.lib().loco_router_backward(cfg, a.get("t", 4), a.get("z", PTR), 8, None, a.get("i", PTR), a.get("c", PTR),
                                                        a.get("l"), a.get("w"), a.get("d", PTR), 8, None)
    assert back(t=-1) == loco.ERR_ARG and back(t=0, z=None) == loco.OK
    for name in ("z", "i", "c", "d"):
        assert back(**{name: None}) == loco.ERR_ARG and back(**{name: PTR + 1}) == loco.ERR_ALIGN
    assert back(l=PTR + 2) == loco.ERR_ALIGN and back(w=PTR + 2) == loco.ERR_ALIGN
