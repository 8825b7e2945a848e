"""The cases on which the operators around a mixture-of-experts layer's products are timed and compared.

What a training step does between the attention, the router and the exchange of gradients:

  norm       root-mean-square norm with the residual's addition, its output in the type of the heads or in 8 bits with
             scales, and the gradient of both
  experts    the router's choices sorted by expert, the tokens laid out in that order and summed back with their weights,
             and the gradient of both ways
  product    the rows of every expert times that expert's matrix, and the gradients of rows and matrices
  clip       the global norm of a list of gradients, and the gradients scaled down to a largest norm

`own` false: plain torch in 32 bits, rounded once at the end.  `own` true: the library's calls.
"""
import math
import random

import torch

own = False

BF16, F32, F64, E4M3 = torch.bfloat16, torch.float32, torch.float64, torch.float8_e4m3fn
DTYPES = {"bf16": BF16, "fp32": F32}
DEV = "cuda"
EPS = 1e-5
E4M3_MAX, LEAST_SCALE = 448.0, 2.0 ** -126


# ------------------------------------------------------------------------------------------------ cases

def listed():
    return [
        # one new token of a 7B decoder on its way into an 8-bit product: nothing but latency
        dict(name="norm, one token, 8 bits", op="norm", rows=1, dim=4096, dtype="bf16", residual=True, weight=True, out="e4m3", block=128),
        # the tokens of four sequences of 4096 in a 13B decoder
        dict(name="norm, 16384 tokens", op="norm", rows=16384, dim=5120, dtype="bf16", residual=True, weight=True, out="same", block=0),
        # an odd width in fp32
        dict(name="norm gradient, odd width, fp32", op="norm gradient", rows=5003, dim=1367, dtype="fp32", residual=True, weight=True),
        # two sequences of 4096 in a 7B decoder
        dict(name="norm gradient, 8192 tokens", op="norm gradient", rows=8192, dim=4096, dtype="bf16", residual=True, weight=True),
        # a handful of tokens: latency of sorting, laying out and summing back
        dict(name="experts, nine tokens", op="experts", tokens=9, dim=4096, experts=8, top_k=2, dtype="bf16", masked=False, weighted=True),
        # a training batch over eight experts, two chosen
        dict(name="experts, 16384 tokens", op="experts", tokens=16384, dim=4096, experts=8, top_k=2, dtype="bf16", masked=False, weighted=True),
        # many experts, padding among the tokens, ragged sizes
        dict(name="experts gradient, 160 experts", op="experts gradient", tokens=5021, dim=2040, experts=160, top_k=6, dtype="bf16", masked=True, weighted=True),
        # four new tokens through the first matrices of eight experts: the matrices' bytes
        dict(name="product, four tokens", op="product", rows=8, d_in=4096, d_out=28672, experts=8, transposed=False, loads=3),
        # a small model's batch over many experts of a few dozen rows each, matrices as a linear layer stores them
        dict(name="product, 64 experts", op="product", rows=3001, d_in=1032, d_out=2048, experts=64, transposed=True, loads=5),
        # 8192 tokens, two choices each, through one matrix of eight experts, and back: the largest
        dict(name="product gradient, 16384 rows", op="product gradient", rows=16384, d_in=4096, d_out=14336, experts=8, transposed=False, loads=7),
        # the tensors of a small model: launches and latency
        dict(name="clip, 37 small tensors", op="clip", tensors=37, total=150001, dtype="mixed", limit=0.5, sizes=11),
        # one of eight ranks' shards of a 7B decoder's 291 gradients
        dict(name="clip, shards of a 7B model", op="clip", tensors=291, total=842000003, dtype="bf16", limit=0.5, sizes=13),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["norm", "norm gradient", "experts", "experts gradient", "product", "product", "product gradient", "clip"])
    if op.startswith("norm"):
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        dim = rng.choice([_log_int(rng, 64, 16384), 8 * _log_int(rng, 8, 2048), 4096, 5120])
        c = dict(op=op, rows=_log_int(rng, 1, max(1, 80_000_000 // dim)), dim=dim, dtype=dtype, residual=rng.random() < 0.7, weight=rng.random() < 0.8)
        if op == "norm":
            c["out"] = rng.choice(["same", "same", "e4m3"])
            c["block"] = rng.choice([0, 128]) if c["out"] == "e4m3" else 0
        return c
    if op.startswith("experts"):
        experts = rng.choice([4, 8, 8, 16, 60, 64, 128, 160, 256])
        top_k = rng.choice([1, 2, 2, 4] + ([6, 8] if experts >= 16 else []))
        dim = rng.choice([_log_int(rng, 64, 8192), 8 * _log_int(rng, 8, 1024), 4096, 2048])
        return dict(op=op, tokens=_log_int(rng, 1, max(1, 130_000_000 // (dim * top_k))), dim=dim, experts=experts, top_k=top_k,
                    dtype=rng.choice(["bf16", "bf16", "fp32"]), masked=rng.random() < 0.4, weighted=rng.random() < 0.8)
    if op.startswith("product"):
        experts = rng.choice([2, 4, 8, 8, 16, 64, 128])
        d_in, d_out = (8 * _log_int(rng, 8, 1792) for _ in range(2))
        experts = max(1, min(experts, 1_000_000_000 // (d_in * d_out)))
        most = int(900e9 / (d_in * d_out)) // (1 if op == "product" else 2)
        return dict(op=op, rows=_log_int(rng, 1, max(1, min(65536, most))), d_in=d_in, d_out=d_out, experts=experts,
                    transposed=rng.random() < 0.5, loads=rng.randint(1, 1 << 20))
    tensors = _log_int(rng, 1, 400)
    return dict(op=op, tensors=tensors, total=_log_int(rng, tensors, 600_000_000), dtype=rng.choice(["bf16", "fp32", "mixed"]),
                limit=rng.choice([0.5, 0.5, 2.0]), sizes=rng.randint(1, 1 << 20))


def _loads(case):
    """Rows of every expert.  Drawn from the case, so that the work is known without the inputs; some experts get more, some none."""
    r, e = random.Random(case["loads"]), case["experts"]
    like = [math.exp(r.gauss(0.0, 0.5)) for _ in range(e)]
    if e > 2 and r.random() < 0.5:
        like[r.randrange(e)] = 0.0
    if case["rows"] < 4 * e:
        n = [0] * e
        for x in r.choices(range(e), like, k=case["rows"]):
            n[x] += 1
        return n
    n = [int(case["rows"] * x / sum(like)) for x in like]
    n[max(range(e), key=lambda i: n[i])] += case["rows"] - sum(n)
    return n


def _sizes(case):
    """Elements of every tensor, from a few to most of the list's."""
    r, k = random.Random(case["sizes"]), case["tensors"]
    like = [math.exp(r.gauss(0.0, 1.5)) for _ in range(k)]
    n = [1 + int((case["total"] - k) * x / sum(like)) for x in like]
    n[max(range(k), key=lambda i: n[i])] += case["total"] - sum(n)
    return n


def _types(case):
    return [F32 if case["dtype"] == "fp32" or case["dtype"] == "mixed" and i % 3 == 2 else BF16 for i in range(case["tensors"])]


def _active(case):
    """Choices that have a row: those of the tokens that are not padding."""
    return (case["tokens"] - (case["tokens"] // 5 if case["masked"] else 0)) * case["top_k"]


# ------------------------------------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _normal(g, shape, dtype=F32, sigma=1.0):
    return torch.randn(shape, generator=g, device=DEV, dtype=F32).mul_(sigma).to(dtype)


def _prepare_norm(c, g):
    n, d, dt = c["rows"], c["dim"], DTYPES[c["dtype"]]
    lean = _normal(g, (d,)).exp_()           # some channels of a residual stream are far larger than others
    st = dict(case=c, x=(_normal(g, (n, d)) * lean).to(dt), r=(_normal(g, (n, d)) * lean).to(dt) if c["residual"] else None,
              w=(1.0 + _normal(g, (d,), sigma=0.2)).to(dt) if c["weight"] else None)
    if c["op"] == "norm":
        e4m3 = c["out"] == "e4m3"
        st["y"] = torch.empty((n, d), dtype=E4M3 if e4m3 else dt, device=DEV)
        st["scale"] = torch.empty((n, -(-d // c["block"]) if c["block"] else 1), dtype=F32, device=DEV) if e4m3 else None
        st["h"] = torch.empty((n, d), dtype=dt, device=DEV) if c["residual"] else None
        return st
    st["dy"] = _normal(g, (n, d), dt, 1e-3)
    st["dh"] = _normal(g, (n, d), dt, 1e-3) if c["residual"] else None
    st["dx"] = torch.empty((n, d), dtype=dt, device=DEV)
    st["dw"] = torch.empty(d, dtype=dt, device=DEV) if c["weight"] else None
    st["work"] = torch.zeros(32 << 20, dtype=torch.uint8, device=DEV)
    return st


def _prepare_experts(c, g):
    t, d, e, k, dt = c["tokens"], c["dim"], c["experts"], c["top_k"], DTYPES[c["dtype"]]
    lean = _normal(g, (e,), sigma=0.7)
    index = torch.topk(_normal(g, (t, e), sigma=1.3) + lean, k, dim=1).indices.to(torch.int32)
    weight = torch.softmax(_normal(g, (t, k)), 1)
    if c["masked"]:                          # padding has no choice
        index[torch.randperm(t, generator=g, device=DEV)[: t // 5]] = -1
    st = dict(case=c, index=index, weight=torch.where(index >= 0, weight, 0.0) if c["weighted"] else None,
              place=torch.empty((t, k), dtype=torch.int32, device=DEV), offsets=torch.empty(e + 1, dtype=torch.int32, device=DEV),
              sort_work=torch.zeros(8 << 20, dtype=torch.uint8, device=DEV))
    st["expert_rows"] = _normal(g, (t * k, d), dt)
    if c["op"] == "experts":
        st["x"] = _normal(g, (t, d), dt)
        st["rows"] = torch.zeros((t * k, d), dtype=dt, device=DEV)
        st["y"] = torch.empty((t, d), dtype=dt, device=DEV)
        return st
    offsets, place = _plain_sort(index, e)
    st["offsets"].copy_(offsets)
    st["place"].copy_(place)
    st["dy"] = _normal(g, (t, d), dt, 1e-3)
    st["drows_in"] = _normal(g, (t * k, d), dt, 1e-3)
    st["drows"] = torch.zeros((t * k, d), dtype=dt, device=DEV)
    st["dweight"] = torch.empty((t, k), dtype=F32, device=DEV) if c["weighted"] else None
    st["dx"] = torch.empty((t, d), dtype=dt, device=DEV)
    return st


def _prepare_product(c, g):
    n, a, b, e = c["rows"], c["d_in"], c["d_out"], c["experts"]
    loads = _loads(c)
    st = dict(case=c, longest=max(loads), offsets=torch.tensor([0] + loads, dtype=torch.int32).cumsum(0).to(torch.int32).to(DEV),
              x=_normal(g, (n, a), BF16))
    st["w"] = torch.empty((e, b, a) if c["transposed"] else (e, a, b), dtype=BF16, device=DEV)
    for i in range(e):
        st["w"][i] = _normal(g, st["w"].shape[1:], BF16, a ** -0.5)
    if c["op"] == "product":
        st["y"] = torch.zeros((n, b), dtype=BF16, device=DEV)
        return st
    st["dy"] = _normal(g, (n, b), BF16, 1e-3)
    st["dx"] = torch.zeros((n, a), dtype=BF16, device=DEV)
    st["dw"] = torch.empty_like(st["w"])
    return st


def _prepare_clip(c, g):
    sizes, types = _sizes(c), _types(c)
    flat = {dt: torch.empty(sum(n for n, t in zip(sizes, types) if t is dt), dtype=dt, device=DEV) for dt in (BF16, F32)}
    out = {dt: torch.empty_like(f) for dt, f in flat.items()}
    at, grads, outs, r = {BF16: 0, F32: 0}, [], [], random.Random(c["sizes"])
    squares = 0.0
    for n, dt in zip(sizes, types):          # tensors one after the other in a flat buffer, each of its own scale
        sigma = 1e-4 * 10.0 ** r.uniform(-1.0, 1.0)
        part = flat[dt][at[dt]:at[dt] + n]
        for lo in range(0, n, 1 << 26):
            part[lo:lo + (1 << 26)] = _normal(g, (min(n - lo, 1 << 26),), dt, sigma)
        grads.append(part)
        outs.append(out[dt][at[dt]:at[dt] + n])
        at[dt] += n
        squares += n * sigma * sigma
    return dict(case=c, grads=grads, outs=outs, flat=[out[dt] for dt in (BF16, F32) if out[dt].numel()], max_norm=c["limit"] * math.sqrt(squares),
                squares=torch.empty(1, dtype=F64, device=DEV), norm=torch.empty(1, dtype=F32, device=DEV),
                work=torch.zeros(1 << 20, dtype=torch.uint8, device=DEV))


def prepare(case, seed):
    g = _gen(seed)
    return {"norm": _prepare_norm, "experts": _prepare_experts, "product": _prepare_product, "clip": _prepare_clip}[case["op"].split()[0]](case, g)


# ------------------------------------------------------------------------------------------------ one pass

def run(state):
    op = state["case"]["op"]
    if own:
        return {"norm": _own_norm, "norm gradient": _own_norm_gradient, "experts": _own_experts, "experts gradient": _own_experts_gradient,
                "product": _own_product, "product gradient": _own_product_gradient, "clip": _own_clip}[op](state)
    return {"norm": _plain_norm, "norm gradient": _plain_norm_gradient, "experts": _plain_experts, "experts gradient": _plain_experts_gradient,
            "product": _plain_product, "product gradient": _plain_product_gradient, "clip": _plain_clip}[op](state)


def _own_norm(st):
    from paper_2407_04480_b200 import layer
    layer.loco_norm_forward(st["x"], st["y"], weight=st["w"], residual=st["r"], total=st["h"], scale=st["scale"], block=st["case"]["block"], eps=EPS)
    return st["y"], st["scale"], st["h"]


def _own_norm_gradient(st):
    from paper_2407_04480_b200 import layer
    layer.loco_norm_backward(st["x"], st["dy"], st["dx"], st["work"], weight=st["w"], dweight=st["dw"], dtotal=st["dh"], eps=EPS)
    return st["dx"], st["dw"]


def _own_experts(st):
    from paper_2407_04480_b200 import layer
    layer.loco_experts_sort(st["index"], st["offsets"], st["place"], st["sort_work"])
    layer.loco_experts_dispatch(st["x"], st["place"], st["rows"])
    layer.loco_experts_combine(st["expert_rows"], st["place"], st["y"], weight=st["weight"])
    return st["offsets"], st["place"], st["rows"], st["y"]


def _own_experts_gradient(st):
    from paper_2407_04480_b200 import layer
    if st["weight"] is None:
        layer.loco_experts_dispatch(st["dy"], st["place"], st["drows"])
    else:
        layer.loco_experts_combine_backward(st["dy"], st["expert_rows"], st["place"], st["weight"], st["drows"], st["dweight"])
    layer.loco_experts_combine(st["drows_in"], st["place"], st["dx"])
    return st["drows"], st["dweight"], st["dx"]


def _own_product(st):
    from paper_2407_04480_b200 import layer
    layer.loco_experts_product(st["x"], st["w"], st["offsets"], st["y"], transposed=st["case"]["transposed"])
    return st["y"]


def _own_product_gradient(st):
    from paper_2407_04480_b200 import layer
    turned = st["case"]["transposed"]
    layer.loco_experts_product(st["dy"], st["w"], st["offsets"], st["dx"], transposed=not turned)
    a, b = (st["dy"], st["x"]) if turned else (st["x"], st["dy"])
    layer.loco_experts_product_weights(a, b, st["offsets"], st["dw"])
    return st["dx"], st["dw"]


def _own_clip(st):
    from paper_2407_04480_b200 import layer
    layer.loco_gradient_squares(st["grads"], st["squares"], st["work"])
    layer.loco_gradient_clip(st["grads"], st["outs"], st["squares"], st["norm"], st["max_norm"])
    return st["norm"], st["flat"]


# plain forms

def _plain_norm(st):
    c, dt = st["case"], st["x"].dtype
    h = st["x"] if st["r"] is None else (st["x"].to(F32) + st["r"].to(F32)).to(dt)
    x = h.to(F32)
    y = x * torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)
    if st["w"] is not None:
        y = y * st["w"].to(F32)
    scale = None
    if c["out"] == "e4m3":
        n, d = y.shape
        block = c["block"] or d
        blocks = -(-d // block)
        part = torch.nn.functional.pad(y, (0, blocks * block - d)).view(n, blocks, block)
        scale = torch.clamp(part.abs().amax(2) / E4M3_MAX, min=LEAST_SCALE)
        y = torch.clamp(part / scale[:, :, None], -E4M3_MAX, E4M3_MAX).view(n, blocks * block)[:, :d]
    return y.to(st["y"].dtype).contiguous(), scale, h if st["r"] is not None else None


def _plain_norm_gradient(st):
    x, dy = st["x"].to(F32), st["dy"].to(F32)
    s = torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)
    unit = x * s
    g = dy if st["w"] is None else dy * st["w"].to(F32)
    dx = s * (g - unit * (g * unit).mean(1, keepdim=True))
    if st["dh"] is not None:
        dx = dx + st["dh"].to(F32)
    return dx.to(st["x"].dtype), None if st["w"] is None else (dy * unit).sum(0).to(st["w"].dtype)


def _plain_sort(index, experts):
    """(offsets, place): the choices in the order of expert, token, slot."""
    flat = index.reshape(-1).long()
    key = torch.where(flat >= 0, flat, experts)
    order = torch.sort(key, stable=True).indices
    row = torch.empty_like(order)
    row[order] = torch.arange(order.numel(), device=order.device)
    ends = torch.zeros(experts + 1, dtype=torch.int64, device=order.device).scatter_add_(0, key, torch.ones_like(key))[:experts].cumsum(0)
    return torch.cat([ends.new_zeros(1), ends]).to(torch.int32), torch.where(flat >= 0, row, -1).to(torch.int32).view(index.shape)


def _spread(values, place, rows):
    """values [tokens, top_k, dim] -> [rows, dim] at their places, zero elsewhere."""
    out = torch.zeros((rows + 1, values.shape[-1]), dtype=values.dtype, device=DEV)
    out[torch.where(place >= 0, place, rows).reshape(-1).long()] = values.reshape(-1, values.shape[-1])
    return out[:rows]


def _at_places(rows, place):
    """fp32 [tokens, top_k, dim]: the rows at their places, zero where there is none."""
    return torch.where((place >= 0)[:, :, None], rows[place.clamp(min=0).long()].to(F32), 0.0)


def _plain_experts(st):
    offsets, place = _plain_sort(st["index"], st["case"]["experts"])
    rows = _spread(st["x"][:, None].expand(-1, place.shape[1], -1), place, st["rows"].shape[0])
    back = _at_places(st["expert_rows"], place)
    if st["weight"] is not None:
        back = back * st["weight"][:, :, None]
    return offsets, place, rows, back.sum(1).to(st["x"].dtype)


def _plain_experts_gradient(st):
    place, dt = st["place"], st["dy"].dtype
    d = st["dy"].to(F32)[:, None].expand(-1, place.shape[1], -1)
    dweight = None
    if st["weight"] is not None:
        dweight = (d * _at_places(st["expert_rows"], place)).sum(2)
        d = d * st["weight"][:, :, None]
    return _spread(d.to(dt), place, st["drows"].shape[0]), dweight, _at_places(st["drows_in"], place).sum(1).to(dt)


def _padded(st, rows):
    """fp32 [experts, longest, dim]: every expert's rows, zero behind them."""
    o, i = st["offsets"].long(), torch.arange(st["longest"], device=DEV)
    there = i < (o[1:] - o[:-1])[:, None]
    return rows[torch.where(there, o[:-1, None] + i, 0)].to(F32) * there[:, :, None]


def _rows(st, padded, like):
    """The inverse, rounded once."""
    o, r = st["offsets"].long(), torch.arange(like.shape[0], device=DEV)
    e = torch.searchsorted(o, r, right=True) - 1
    return padded[e, r - o[e]].to(like.dtype)


def _plain_product(st):
    w = st["w"].to(F32)
    return _rows(st, torch.matmul(_padded(st, st["x"]), w.transpose(1, 2) if st["case"]["transposed"] else w), st["y"])


def _plain_product_gradient(st):
    w, turned = st["w"].to(F32), st["case"]["transposed"]
    x, dy = _padded(st, st["x"]), _padded(st, st["dy"])
    dx = _rows(st, torch.matmul(dy, w if turned else w.transpose(1, 2)), st["dx"])
    a, b = (dy, x) if turned else (x, dy)
    return dx, torch.matmul(a.transpose(1, 2), b).to(BF16)


def _plain_clip(st):
    norm = torch.sqrt(torch.stack([x.to(F64).square().sum() for x in st["grads"]]).sum())
    by = torch.where(norm > st["max_norm"], st["max_norm"] / norm, 1.0).to(F32)
    _ = [o.copy_(x.to(F32) * by) for x, o in zip(st["grads"], st["outs"])]
    return norm.to(F32).reshape(1), st["flat"]


# ------------------------------------------------------------------------------------------------ work

def work(case):
    c = case
    size = 4 if c.get("dtype") == "fp32" else 2
    if c["op"] == "norm":
        out = 1 if c["out"] == "e4m3" else size
        scales = 4 * c["rows"] * (-(-c["dim"] // c["block"]) if c["block"] else 1) if c["out"] == "e4m3" else 0
        return {"bytes": c["rows"] * c["dim"] * (size * (3 if c["residual"] else 1) + out) + scales + (size * c["dim"] if c["weight"] else 0),
                "flops": 5 * c["rows"] * c["dim"]}
    if c["op"] == "norm gradient":
        return {"bytes": c["rows"] * c["dim"] * size * (4 if c["residual"] else 3) + (2 * size * c["dim"] if c["weight"] else 0),
                "flops": 10 * c["rows"] * c["dim"]}
    if c["op"] == "experts":
        t, a = c["tokens"], _active(c)
        return {"bytes": 2 * (t + a) * c["dim"] * size + t * c["top_k"] * (12 if c["weighted"] else 8) + 4 * (c["experts"] + 1),
                "flops": 2 * a * c["dim"]}
    if c["op"] == "experts gradient":
        t, a, w = c["tokens"], _active(c), c["weighted"]
        return {"bytes": (2 * t + (3 if w else 2) * a) * c["dim"] * size + t * c["top_k"] * (12 if w else 4), "flops": (4 if w else 1) * a * c["dim"]}
    if c["op"].startswith("product"):
        n, a, b = c["rows"], c["d_in"], c["d_out"]
        live = sum(x > 0 for x in _loads(c))
        if c["op"] == "product":
            return {"bytes": 2 * (n * (a + b) + live * a * b), "flops": 2 * n * a * b}
        return {"bytes": 2 * (n * (a + b) + n * a + (live + c["experts"]) * a * b), "flops": 4 * n * a * b}
    return {"bytes": sum(2 * n * (4 if t is F32 else 2) for n, t in zip(_sizes(c), _types(c))), "flops": 3 * c["total"]}


# ------------------------------------------------------------------------------------------------ 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    return {"norm": _exact_norm, "norm gradient": _exact_norm_gradient, "experts": _exact_experts, "experts gradient": _exact_experts_gradient,
            "product": _exact_product, "product gradient": _exact_product_gradient, "clip": _exact_clip}[case["op"]](st)


def _unit(h, w):
    y = h / torch.sqrt(h.square().sum(1, keepdim=True) / h.shape[1] + EPS)
    return y if w is None else y * w


def _exact_norm(st):
    c, dt = st["case"], st["x"].dtype
    h = st["x"].double()
    if st["r"] is not None:                  # the sum as it is kept: in the type of the heads
        h = (h + st["r"].double()).to(dt).double()
    y = _unit(h, None if st["w"] is None else st["w"].double())
    scale = None
    if c["out"] == "e4m3":
        step = c["block"] or c["dim"]
        cuts = range(0, c["dim"], step)
        scale = torch.stack([(y[:, i:i + step].abs().amax(1) / E4M3_MAX).clamp(min=LEAST_SCALE) for i in cuts], 1)
        y = torch.cat([(y[:, i:i + step] / scale[:, j:j + 1]).to(F32).to(E4M3).double() for j, i in enumerate(cuts)], 1)
    return y, scale, h if st["r"] is not None else None


def _exact_norm_gradient(st):
    """By torch's differentiation, a few thousand rows at a time."""
    w = None if st["w"] is None else st["w"].double().requires_grad_()
    dx, dw = [], None if w is None else torch.zeros_like(w)
    for x, dy in zip(st["x"].split(4096), st["dy"].split(4096)):
        h = x.double().requires_grad_()
        got = torch.autograd.grad(_unit(h, w), [h] + ([] if w is None else [w]), dy.double())
        dx.append(got[0])
        if w is not None:
            dw = dw + got[1]
    dx = torch.cat(dx)
    return dx if st["dh"] is None else dx + st["dh"].double(), dw


def _exact_experts(st):
    """Choice by choice: where every expert's turn comes is counted on the host."""
    c = st["case"]
    index = st["index"].cpu().numpy().reshape(-1)
    count = [0] * c["experts"]
    for e in index[index >= 0].tolist():
        count[e] += 1
    first = [0]
    for n in count:
        first.append(first[-1] + n)
    at, place = list(first), []
    for e in index.tolist():
        place.append(at[e] if e >= 0 else -1)
        if e >= 0:
            at[e] += 1
    place = torch.tensor(place, dtype=torch.int32, device=DEV).view(st["index"].shape)
    rows = torch.zeros(st["rows"].shape, dtype=F64, device=DEV)
    y = torch.zeros(st["x"].shape, dtype=F64, device=DEV)
    for j in range(c["top_k"]):
        some = place[:, j] >= 0
        p = place[some, j].long()
        rows[p] = st["x"][some].double()
        y[some] += st["expert_rows"][p].double() * (1.0 if st["weight"] is None else st["weight"][some, j:j + 1].double())
    return torch.tensor(first, dtype=torch.int32, device=DEV), place, rows, y


def _exact_experts_gradient(st):
    c, place = st["case"], st["place"]
    drows = torch.zeros(st["drows"].shape, dtype=F64, device=DEV)
    dx = torch.zeros(st["dy"].shape, dtype=F64, device=DEV)
    dweight = None if st["weight"] is None else torch.zeros(place.shape, dtype=F64, device=DEV)
    for j in range(c["top_k"]):
        some = place[:, j] >= 0
        p, d = place[some, j].long(), st["dy"][some].double()
        if dweight is not None:
            dweight[some, j] = torch.einsum("td,td->t", d, st["expert_rows"][p].double())
            d = d * st["weight"][some, j:j + 1].double()
        drows[p] = d
        dx[some] += st["drows_in"][p].double()
    return drows, dweight, dx


def _by_expert(st):
    """(expert, its rows) of every expert that has some."""
    at = 0
    for e, n in enumerate(_loads(st["case"])):
        if n:
            yield e, slice(at, at + n)
        at += n


def _exact_product(st):
    y = torch.zeros(st["y"].shape, dtype=F64, device=DEV)
    for e, rows in _by_expert(st):
        w = st["w"][e].double()
        y[rows] = st["x"][rows].double() @ (w.T if st["case"]["transposed"] else w)
    return y


def _exact_product_gradient(st):
    dx, dw = (torch.zeros(st[x].shape, dtype=F64, device=DEV) for x in ("dx", "dw"))
    for e, rows in _by_expert(st):
        w, x, dy = st["w"][e].double(), st["x"][rows].double(), st["dy"][rows].double()
        if st["case"]["transposed"]:
            dx[rows], dw[e] = dy @ w, dy.T @ x
        else:
            dx[rows], dw[e] = dy @ w.T, x.T @ dy
    return dx, dw


def _exact_clip(st):
    norm = math.sqrt(math.fsum(float(torch.dot(p, p)) for x in st["grads"] for p in x.double().split(1 << 27)))
    by = st["max_norm"] / norm if norm > st["max_norm"] else 1.0
    flat = [torch.cat([x.double() * by for x in st["grads"] if x.dtype == f.dtype]) for f in st["flat"]]
    return torch.tensor([norm], dtype=F64, device=DEV), flat
