"""The cases on which the operators of a decoder layer's training step are timed and compared.

Three operators and their gradients, as a data-parallel trainer runs them before its gradients are compressed:

  rotary     rotary positions on the query and key heads, and the transposed rotation of their gradients
  attention  softmax attention (bf16, grouped heads, causal, padded or packed sequences): the forward pass, which
             leaves the log-sum-exp of every row, and the backward pass, which recomputes the probabilities from it
  router     a mixture-of-experts router: the chosen experts and their weights, per-expert counts, the balance and
             the z loss, and the gradient of all of them with respect to the logits

`own` false: plain torch in 32 bits, rounded once at the end.  `own` true: the library's calls.
"""
import math
import random

import torch

own = False

BF16, F32 = torch.bfloat16, torch.float32
DTYPES = {"bf16": BF16, "fp32": F32}
DEV = "cuda"


# ------------------------------------------------------------------------------------------------ cases

def listed():
    return [
        # one new token of a decoder with 8 shared key heads: nothing but latency
        dict(name="rotary, one token", op="rotary", batch=1, seq=1, heads_q=32, heads_k=8, head_dim=128, rotary_dim=128,
             layout="half", dtype="bf16", inverse=False, fused=False, positions="given", scaling="none"),
        # fp32 heads of odd width, a part of which is rotated, cut out of one projection's output, ragged length, context
        # stretched eight times by parts
        dict(name="rotary, part of odd heads, fp32", op="rotary", batch=3, seq=1367, heads_q=16, heads_k=16, head_dim=80,
             rotary_dim=32, layout="interleaved", dtype="fp32", inverse=False, fused=True, positions="given", scaling="parts"),
        # the gradients of the query and key heads of a 7B decoder, four sequences of 4096
        dict(name="rotary, gradient, 7B heads", op="rotary", batch=4, seq=4096, heads_q=32, heads_k=32, head_dim=128,
             rotary_dim=128, layout="half", dtype="bf16", inverse=True, fused=False, positions="implicit", scaling="none"),
        # a short unmasked sequence of a small model: latency
        dict(name="attention, short", op="attention", batch=1, seq_q=77, seq_k=77, heads_q=16, heads_kv=16, head_dim=64,
             causal=False, form="padded", lens=0, fused=False),
        # two sequences of 4096 in one layer with 32 query and 8 key heads, straight from the fused projection
        dict(name="attention, 4096, grouped", op="attention", batch=2, seq_q=4096, seq_k=4096, heads_q=32, heads_kv=8,
             head_dim=128, causal=True, form="padded", lens=0, fused=True),
        # instruction samples of very different lengths packed into one row
        dict(name="attention, packed", op="attention", batch=13, seq_q=611, seq_k=611, heads_q=32, heads_kv=8, head_dim=128,
             causal=True, form="packed", lens=5, fused=False),
        # a padded batch of a small bidirectional model with an empty sample in it
        dict(name="attention gradient, padded", op="gradient", batch=4, seq_q=197, seq_k=197, heads_q=16, heads_kv=16,
             head_dim=64, causal=False, form="padded", lens=3, fused=False),
        # the packed instruction samples' gradient
        dict(name="attention gradient, packed", op="gradient", batch=11, seq_q=727, seq_k=727, heads_q=32, heads_kv=8,
             head_dim=128, causal=True, form="packed", lens=7, fused=False),
        # one long sequence through all 32 heads of a 7B layer: the largest
        dict(name="attention gradient, 8192", op="gradient", batch=1, seq_q=8192, seq_k=8192, heads_q=32, heads_kv=32,
             head_dim=128, causal=True, form="padded", lens=0, fused=False),
        # a handful of tokens: latency of the whole router step
        dict(name="router, nine tokens", op="router", tokens=9, experts=8, top_k=2, dtype="bf16", normalize=True, masked=False),
        # a batch of 32768 tokens over eight experts, two chosen
        dict(name="router, 8 experts", op="router", tokens=32768, experts=8, top_k=2, dtype="bf16", normalize=True, masked=False),
        # many experts, padding among the tokens, fp32 logits, weights that are not normalised
        dict(name="router, 160 experts", op="router", tokens=50021, experts=160, top_k=6, dtype="fp32", normalize=False, masked=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["rotary", "attention", "gradient", "gradient", "router"])
    if op == "rotary":
        head_dim = rng.choice([64, 80, 96, 128, 128, 36])
        heads_k = rng.choice([1, 2, 8, 16])
        heads_q = heads_k * rng.choice([1, 2, 4])
        batch = rng.randint(1, 4)
        return dict(op=op, batch=batch, seq=_log_int(rng, 1, 16384 // batch), heads_q=heads_q, heads_k=heads_k, head_dim=head_dim,
                    rotary_dim=rng.choice([head_dim, head_dim // 4 * 2, 16]), layout=rng.choice(["half", "interleaved"]),
                    dtype=rng.choice(["bf16", "bf16", "fp32"]), inverse=rng.random() < 0.5, fused=rng.random() < 0.5,
                    positions=rng.choice(["implicit", "given"]), scaling=rng.choice(["none", "linear", "parts"]))
    if op == "router":
        experts = rng.choice([4, 8, 8, 16, 60, 64, 128, 160, 256])
        return dict(op=op, tokens=_log_int(rng, 1, 131072 if experts <= 64 else 40000), experts=experts,
                    top_k=rng.choice([1, 2, 2, 4] + ([6, 8] if experts >= 16 else [])), dtype=rng.choice(["bf16", "fp32"]),
                    normalize=rng.random() < 0.6, masked=rng.random() < 0.4)
    batch = rng.choice([1, 1, 2, 3, 7, 16])
    heads_kv = rng.choice([1, 2, 8, 16])
    heads_q = heads_kv * rng.choice([1, 1, 2, 4] if heads_kv < 16 else [1, 2])
    most = int(math.sqrt(32 * 8192 * 8192 / (batch * heads_q)))
    seq_q = _log_int(rng, 1, min(8192, most))
    form = rng.choice(["padded", "padded", "packed"])
    seq_k = seq_q if form == "packed" or rng.random() < 0.7 else _log_int(rng, 1, min(8192, max(1, 32 * 8192 * 8192 // (batch * heads_q * max(seq_q, 1024)))))
    return dict(op=op, batch=batch, seq_q=seq_q, seq_k=seq_k, heads_q=heads_q, heads_kv=heads_kv,
                head_dim=rng.choice([64, 64, 128, 128, 128, 96, 40]), causal=rng.random() < 0.6, form=form,
                lens=rng.randint(1, 1 << 20) if form == "packed" or rng.random() < 0.3 else 0, fused=seq_q == seq_k and rng.random() < 0.3)


def _lengths(case):
    """Per sample: (query length, key length).  Drawn from the case, so that the work is known without the inputs."""
    b, sq, sk = case["batch"], case["seq_q"], case["seq_k"]
    if not case["lens"]:
        return [sq] * b, [sk] * b
    r = random.Random(case["lens"])
    if case["form"] == "packed":             # cuts of one row of batch * seq tokens
        total = b * sq
        cuts = sorted(r.randint(0, total) for _ in range(b - 1))
        n = [hi - lo for lo, hi in zip([0] + cuts, cuts + [total])]
        return n, n
    nk = [r.randint(1, sk) for _ in range(b)]
    if b > 2:
        nk[r.randrange(b)] = 0               # an empty sample
    nk[r.randrange(b)] = sk
    return (list(nk) if sq == sk else [sq] * b), nk


# ------------------------------------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _normal(g, shape, dtype=F32, sigma=1.0):
    return (torch.randn(shape, generator=g, device=DEV, dtype=F32) * sigma).to(dtype)


def _frequencies(r, scaling):
    """Angular frequencies of a rotated part of r dimensions, base 10000, in 64 bits."""
    j = torch.arange(r // 2, dtype=torch.float64)
    w = 10000.0 ** (-2.0 * j / r)
    if scaling == "linear":                  # positions divided by four
        w = w / 4.0
    elif scaling == "parts":                 # context stretched eight times from 4096: slow dimensions divided, fast ones kept
        turns = 4096.0 * w / (2.0 * math.pi)
        keep = ((turns - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
        w = w / 8.0 * (1.0 - keep) + w * keep
    return w


def _prepare_rotary(c, g):
    b, s, hq, hk, d, r = c["batch"], c["seq"], c["heads_q"], c["heads_k"], c["head_dim"], c["rotary_dim"]
    dt = DTYPES[c["dtype"]]
    rows = s if c["positions"] == "implicit" else max(4 * s, 4096)
    if c["fused"]:                           # heads of one projection's output: queries, keys, values
        qkv = _normal(g, (b, s, hq + 2 * hk, d), dt)
        q, k = qkv[:, :, :hq], qkv[:, :, hq:hq + hk]
    else:
        q, k = _normal(g, (b, s, hq, d), dt), _normal(g, (b, s, hk, d), dt)
    angle = torch.outer(torch.arange(rows, dtype=torch.float64), _frequencies(r, c["scaling"])).to(DEV)
    grow = 0.1 * math.log(8.0) + 1.0 if c["scaling"] == "parts" else 1.0
    table = torch.cat([torch.cos(angle) * grow, torch.sin(angle) * grow], 1).to(F32)
    pos = None
    if c["positions"] == "given":            # every sample starts somewhere else
        at = torch.randint(0, rows - s + 1, (b, 1), generator=g, device=DEV)
        pos = (at + torch.arange(s, device=DEV)).to(torch.int32)
    return dict(case=c, q=q, k=k, table=table, positions=pos, q_out=torch.empty((b, s, hq, d), dtype=dt, device=DEV),
                k_out=torch.empty((b, s, hk, d), dtype=dt, device=DEV))


def _prepare_attention(c, g):
    b, sq, sk, hq, hk, d = (c[x] for x in ("batch", "seq_q", "seq_k", "heads_q", "heads_kv", "head_dim"))
    nq, nk = _lengths(c)
    ragged, packed = bool(c["lens"]), c["form"] == "packed"
    rq, rk = ((b * sq,), (b * sk,)) if packed else ((b, sq), (b, sk))
    if c["fused"]:
        qkv = _normal(g, (*rq, hq + 2 * hk, d), BF16)
        q, k, v = qkv[..., :hq, :], qkv[..., hq:hq + hk, :], qkv[..., hq + hk:, :]
    else:
        q, k, v = _normal(g, (*rq, hq, d), BF16), _normal(g, (*rk, hk, d), BF16), _normal(g, (*rk, hk, d), BF16)
    do = _normal(g, (*rq, hq, d), BF16)
    st = dict(case=c, q=q, k=k, v=v, do=do, len_q=None, len_k=None, cu_q=None, cu_k=None, max_q=max(nq), max_k=max(nk))
    if packed:
        cu = torch.tensor([0] + nq, dtype=torch.int32).cumsum(0).to(torch.int32).to(DEV)
        st["cu_q"] = st["cu_k"] = cu
    elif ragged:                             # what lies past a sample's length is whatever the buffer held before
        st["len_q"], st["len_k"] = (torch.tensor(n, dtype=torch.int32, device=DEV) for n in (nq, nk))
        for t, n in ((q, st["len_q"]), (do, st["len_q"]), (k, st["len_k"]), (v, st["len_k"])):
            t[torch.arange(t.shape[1], device=DEV)[None, :] >= n[:, None].long()] = float("nan")
    st["o"] = torch.empty(q.shape, dtype=BF16, device=DEV)
    st["lse"] = torch.empty((hq, b * sq) if packed else (b, hq, sq), dtype=F32, device=DEV)
    if c["op"] == "gradient":
        o, lse = _plain_attention(st)
        st["o"].copy_(o)
        st["lse"].copy_(lse)
        for name, like in (("dq", q), ("dk", k), ("dv", v)):
            st[name] = torch.empty(like.shape, dtype=BF16, device=DEV)
        # fp32 row sums of the gradient pass and its status word
        st["work"] = torch.empty(4 * hq * b * sq + 256, dtype=torch.uint8, device=DEV)
    return st


def _prepare_router(c, g):
    t, e = c["tokens"], c["experts"]
    lean = _normal(g, (e,), sigma=0.7)       # some experts are liked more than others, some hardly at all
    lean[torch.randperm(e, generator=g, device=DEV)[: max(1, e // 4)]] -= 4.0
    z = (_normal(g, (t, e), sigma=1.3) + lean).to(DTYPES[c["dtype"]])
    mask = (torch.rand(t, generator=g, device=DEV) < 0.8).to(torch.uint8) if c["masked"] else None
    k = c["top_k"]
    return dict(case=c, logits=z, mask=mask, dweights=_normal(g, (t, k), sigma=1e-3),
                dlosses=torch.rand(2, generator=g, device=DEV) + 0.5,
                index=torch.empty((t, k), dtype=torch.int32, device=DEV), weights=torch.empty((t, k), dtype=F32, device=DEV),
                counts=torch.empty(e + 1, dtype=torch.int32, device=DEV), mean=torch.empty(e, dtype=F32, device=DEV),
                losses=torch.empty(2, dtype=F32, device=DEV), dlogits=torch.empty_like(z),
                work=torch.zeros(2 << 20, dtype=torch.uint8, device=DEV))


def prepare(case, seed):
    g = _gen(seed)
    return {"rotary": _prepare_rotary, "attention": _prepare_attention, "gradient": _prepare_attention,
            "router": _prepare_router}[case["op"]](case, g)


# ------------------------------------------------------------------------------------------------ one pass

BALANCE, ZLOSS = 0.01, 0.001


def run(state):
    op = state["case"]["op"]
    if own:
        return {"rotary": _own_rotary, "attention": _own_attention, "gradient": _own_gradient, "router": _own_router}[op](state)
    return {"rotary": _plain_rotary, "attention": _plain_attention, "gradient": _plain_gradient, "router": _plain_router}[op](state)


def _own_rotary(st):
    from paper_2407_04480_b200 import layer
    c = st["case"]
    layer.loco_rotary_apply(st["table"], st["q"], st["k"], st["q_out"], st["k_out"], positions=st["positions"],
                            layout=c["layout"], inverse=c["inverse"])
    return st["q_out"], st["k_out"]


def _lens(st):
    return {x: st[x] for x in ("len_q", "len_k", "cu_q", "cu_k", "max_q", "max_k")}


def _own_attention(st):
    from paper_2407_04480_b200 import layer
    layer.loco_attention_forward(st["q"], st["k"], st["v"], st["o"], st["lse"], causal=st["case"]["causal"], **_lens(st))
    return st["o"], st["lse"]


def _own_gradient(st):
    from paper_2407_04480_b200 import layer
    layer.loco_attention_backward(st["q"], st["k"], st["v"], st["o"], st["lse"], st["do"], st["dq"], st["dk"], st["dv"],
                                  st["work"], causal=st["case"]["causal"], **_lens(st))
    return st["dq"], st["dk"], st["dv"]


def _own_router(st):
    from paper_2407_04480_b200 import layer
    c = st["case"]
    cfg = layer.Router(experts=c["experts"], top_k=c["top_k"], normalize=c["normalize"], balance_coef=BALANCE, z_coef=ZLOSS)
    layer.loco_router_forward(cfg, st["logits"], st["index"], st["weights"], st["counts"], st["mean"], st["losses"], st["work"],
                              mask=st["mask"])
    layer.loco_router_backward(cfg, st["logits"], st["index"], st["counts"], st["dlogits"], mask=st["mask"],
                               dlosses=st["dlosses"], dweights=st["dweights"])
    return {x: st[x] for x in ("index", "weights", "counts", "mean", "losses", "dlogits")}


# plain forms

def _plain_rotary(st):
    c, table = st["case"], st["table"]
    r, h = c["rotary_dim"], c["rotary_dim"] // 2
    pos = torch.arange(c["seq"], device=DEV).expand(c["batch"], -1) if st["positions"] is None else st["positions"].long()
    cos, sin = table[pos, None, :h], table[pos, None, h:]
    if c["inverse"]:
        sin = -sin

    def turn(x):
        y = x.to(F32).clone()
        a, b = (slice(0, h), slice(h, r)) if c["layout"] == "half" else (slice(0, r, 2), slice(1, r, 2))
        xa, xb = y[..., a], y[..., b]
        ya, yb = xa * cos - xb * sin, xb * cos + xa * sin
        y[..., a], y[..., b] = ya, yb
        return y.to(x.dtype)
    return turn(st["q"]), turn(st["k"])


def _rows(st):
    """Padded places of every sample: ((index into the rows, validity) of queries, of keys), each [batch, longest]."""
    c = st["case"]
    b = c["batch"]

    def places(cu, n, seq, longest):
        i = torch.arange(longest, device=DEV)[None, :]
        if cu is not None:
            ok = i < (cu[1:] - cu[:-1])[:, None]
            return torch.where(ok, cu[:-1, None] + i, 0).long(), ok
        at = torch.arange(b, device=DEV)[:, None] * seq + i
        return at, (torch.ones_like(at, dtype=torch.bool) if n is None else i < n[:, None])
    packed = c["form"] == "packed"
    return (places(st["cu_q"], st["len_q"], c["seq_q"], st["max_q"] if packed else c["seq_q"]),
            places(st["cu_k"], st["len_k"], c["seq_k"], st["max_k"] if packed else c["seq_k"]))


def _spread(x, at, ok):
    """[..., heads, dim] rows -> fp32 [batch, heads, longest, dim], zero where nothing is."""
    x = x.reshape(-1, *x.shape[-2:])[at].to(F32)
    return torch.where(ok[..., None, None], x, 0.0).transpose(1, 2)


def _gather(y, at, ok, like):
    """The inverse: fp32 [batch, heads, longest, dim] -> rows shaped as `like`, rounded once."""
    rows = torch.zeros((like.shape[:-2].numel(), *like.shape[-2:]), dtype=like.dtype, device=DEV)
    rows[at[ok]] = y.transpose(1, 2)[ok].to(like.dtype)
    return rows.reshape(like.shape)


def _scores(st, q, k, okq, okk):
    c = st["case"]
    s = torch.matmul(q, k.transpose(-1, -2)) * (1.0 / math.sqrt(c["head_dim"]))
    see = okq[:, None, :, None] & okk[:, None, None, :]
    if c["causal"]:
        i, j = torch.arange(okq.shape[1], device=DEV), torch.arange(okk.shape[1], device=DEV)
        off = okk.sum(1) - okq.sum(1)
        see = see & (j[None, :] <= i[:, None] + off[:, None, None])[:, None]
    return s.masked_fill_(~see, float("-inf"))


def _plain_attention(st):
    c = st["case"]
    (aq, okq), (ak, okk) = _rows(st)
    group = c["heads_q"] // c["heads_kv"]
    q = _spread(st["q"], aq, okq)
    k, v = (_spread(st[x], ak, okk).repeat_interleave(group, 1) for x in "kv")
    s = _scores(st, q, k, okq, okk)
    top = s.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), 0.0, top)
    p = torch.exp(s - top)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total > 0, total, 1.0)
    lse = (torch.log(total) + top)[..., 0]
    if c["form"] == "packed":
        out = torch.full(st["lse"].shape, float("-inf"), device=DEV)
        out[:, aq[okq]] = lse.transpose(0, 1)[:, okq]
        lse = out
    return _gather(o, aq, okq, st["q"]), lse


def _plain_gradient(st):
    c = st["case"]
    (aq, okq), (ak, okk) = _rows(st)
    group, hk = c["heads_q"] // c["heads_kv"], c["heads_kv"]
    q, do, o = (_spread(st[x], aq, okq) for x in ("q", "do", "o"))
    k, v = (_spread(st[x], ak, okk).repeat_interleave(group, 1) for x in "kv")
    lse = st["lse"][:, aq].transpose(0, 1) if c["form"] == "packed" else st["lse"]
    some = ~torch.isinf(lse)[..., None]
    p = torch.where(some, torch.exp(_scores(st, q, k, okq, okk) - torch.where(some, lse[..., None], 0.0)), 0.0)
    dv = torch.matmul(p.transpose(-1, -2), do)
    ds = torch.matmul(do, v.transpose(-1, -2)).sub_((do * o).sum(-1, keepdim=True)).mul_(p)
    del p
    scale = 1.0 / math.sqrt(c["head_dim"])
    dq = torch.matmul(ds, k) * scale
    dk = torch.matmul(ds.transpose(-1, -2), q) * scale
    dk, dv = (x.unflatten(1, (hk, group)).sum(2) for x in (dk, dv))
    return _gather(dq, aq, okq, st["q"]), _gather(dk, ak, okk, st["k"]), _gather(dv, ak, okk, st["v"])


def _plain_router(st):
    c = st["case"]
    e, k = c["experts"], c["top_k"]
    z = st["logits"].to(F32)
    there = z != float("-inf")
    active = there.any(1)
    if st["mask"] is not None:
        active = active & (st["mask"] != 0)
    there = there & active[:, None]
    z = torch.where(there, z, float("-inf"))
    top = torch.where(active, z.amax(1), 0.0)[:, None]
    x = torch.exp(z - top)
    total = torch.where(active, x.sum(1), 1.0)[:, None]
    p = x / total
    lse = torch.where(active, (torch.log(total) + top)[:, 0], 0.0)
    order = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :k]
    chosen = torch.gather(there, 1, order)
    index = torch.where(chosen, order, -1).to(torch.int32)
    w = torch.where(chosen, torch.gather(p, 1, order), 0.0)
    share = w.sum(1, keepdim=True) if c["normalize"] else torch.ones_like(total)
    share = torch.where(share > 0, share, 1.0)
    weights = w / share
    counts = torch.zeros(e + 1, dtype=torch.int32, device=DEV)
    counts.scatter_add_(0, torch.where(chosen, order, e).reshape(-1), torch.ones(order.numel(), dtype=torch.int32, device=DEV))
    counts[e] = active.sum()
    n = counts[e].clamp(min=1).to(F32)
    mean = p.sum(0) / n
    load = counts[:e].to(F32) / (n * k)
    losses = torch.stack([BALANCE * e * (load * mean).sum(), ZLOSS * (lse * lse).sum() / n])
    # gradient
    gl = st["dlosses"]
    gp = (gl[0] * BALANCE * e) * load / n
    dz = p * (gp - (p * gp).sum(1, keepdim=True)) + (gl[1] * ZLOSS * 2.0 / n) * lse[:, None] * p
    dw = torch.where(chosen, st["dweights"], 0.0)
    if c["normalize"]:
        dz = dz.scatter_add(1, order, weights * (dw - (weights * dw).sum(1, keepdim=True)))
    else:
        dz = dz.scatter_add(1, order, w * dw) - p * (w * dw).sum(1, keepdim=True)
    dz = torch.where(there, dz, 0.0)
    return {"index": index, "weights": weights, "counts": counts, "mean": mean, "losses": losses,
            "dlogits": dz.to(st["logits"].dtype)}


# ------------------------------------------------------------------------------------------------ work

def work(case):
    c = case
    if c["op"] == "rotary":
        size = 4 if c["dtype"] == "fp32" else 2
        t = c["batch"] * c["seq"]
        heads = c["heads_q"] + c["heads_k"]
        rows = c["seq"] if c["positions"] == "implicit" else t
        return {"bytes": 2 * t * heads * c["head_dim"] * size + 4 * rows * c["rotary_dim"] + (4 * t if c["positions"] == "given" else 0),
                "flops": 3 * t * heads * c["rotary_dim"]}
    if c["op"] == "router":
        t, e, k = c["tokens"], c["experts"], c["top_k"]
        size = 4 if c["dtype"] == "fp32" else 2
        return {"bytes": 2 * t * e * size + t * k * 12 + (t if c["masked"] else 0) + 8 * e, "flops": 12 * t * e}
    nq, nk = _lengths(c)
    if c["form"] == "padded" and not c["lens"]:
        nq, nk = [c["seq_q"]] * c["batch"], [c["seq_k"]] * c["batch"]
    pairs = sum(_pairs(a, b, c["causal"]) for a, b in zip(nq, nk))
    rq, rk = sum(nq), sum(nk)
    d, hq, hk = c["head_dim"], c["heads_q"], c["heads_kv"]
    if c["op"] == "attention":
        return {"bytes": 2 * d * (2 * rq * hq + 2 * rk * hk) + 4 * rq * hq, "flops": 4 * pairs * hq * d}
    return {"bytes": 2 * d * (4 * rq * hq + 4 * rk * hk) + 4 * rq * hq, "flops": 10 * pairs * hq * d}


def _pairs(nq, nk, causal):
    """Query-key pairs that take part."""
    if not causal:
        return nq * nk
    first = max(0, nq - nk)                  # rows before the diagonal enters see nothing
    n = nq - first
    return n * (nk - nq + first + 1) + n * (n - 1) // 2


# ------------------------------------------------------------------------------------------------ 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "rotary":
        return _exact_rotary(st)
    if case["op"] == "router":
        return _exact_router(st)
    return _exact_attention(st)


def _exact_rotary(st):
    """Each pair as a complex number times the table's complex number."""
    c = st["case"]
    r, h = c["rotary_dim"], c["rotary_dim"] // 2
    pos = torch.arange(c["seq"], device=DEV)[None].expand(c["batch"], -1) if st["positions"] is None else st["positions"].long()
    turn = torch.complex(st["table"][pos][..., :h].double(), st["table"][pos][..., h:].double())[:, :, None]
    if c["inverse"]:
        turn = turn.conj()
    out = []
    for x in (st["q"], st["k"]):
        y = x.double()
        part = y[..., :r].unflatten(-1, (2, h)).transpose(-1, -2) if c["layout"] == "half" else y[..., :r].unflatten(-1, (h, 2))
        z = torch.view_as_real(torch.view_as_complex(part.contiguous()) * turn)
        z = (z.transpose(-1, -2) if c["layout"] == "half" else z).flatten(-2)
        out.append(torch.cat([z, y[..., r:]], -1))
    return tuple(out)


def _exact_attention(st):
    """Sample by sample and head by head; the gradient by torch's differentiation of softmax(q k^T) v."""
    c = st["case"]
    nq, nk = _lengths(c)
    packed, grad = c["form"] == "packed", c["op"] == "gradient"
    hq, group, d = c["heads_q"], c["heads_q"] // c["heads_kv"], c["head_dim"]
    f64 = torch.float64
    flat = {x: st[x].reshape(-1, *st[x].shape[-2:]) for x in ("q", "k", "v", "do")}
    res = {x: torch.zeros(flat[y].shape, dtype=f64, device=DEV) for x, y in (("o", "q"), ("dq", "q"), ("dk", "k"), ("dv", "v"))}
    lse = torch.full(st["lse"].shape, float("-inf"), dtype=f64, device=DEV)
    sq = sk = 0
    for b in range(c["batch"]):
        if not packed:
            sq, sk = b * c["seq_q"], b * c["seq_k"]
        rq, rk = slice(sq, sq + nq[b]), slice(sk, sk + nk[b])
        skip = max(0, nq[b] - nk[b]) if c["causal"] else 0            # rows that see no key
        if nk[b] and nq[b] > skip:
            for h in range(hq):
                q, do = (flat[x][rq, h].double()[skip:] for x in ("q", "do"))
                k, v = (flat[x][rk, h // group].double() for x in "kv")
                if grad:
                    q, k, v = (x.requires_grad_() for x in (q, k, v))
                s = q @ k.T / math.sqrt(d)
                if c["causal"]:
                    s = s.masked_fill(torch.ones_like(s, dtype=torch.bool).triu(1 + nk[b] - nq[b] + skip), float("-inf"))
                o = torch.softmax(s, -1) @ v
                at = slice(sq + skip, sq + nq[b])
                if grad:
                    gq, gk, gv = torch.autograd.grad(o, (q, k, v), do)
                    res["dq"][at, h] = gq
                    res["dk"][rk, h // group] += gk
                    res["dv"][rk, h // group] += gv
                else:
                    res["o"][at, h] = o
                    row = torch.logsumexp(s, -1)
                    if packed:
                        lse[h, at] = row
                    else:
                        lse[b, h, skip:nq[b]] = row
        sq, sk = sq + nq[b], sk + nk[b]
    if grad:
        return tuple(res[x].reshape(st[y].shape) for x, y in (("dq", "q"), ("dk", "k"), ("dv", "v")))
    return res["o"].reshape(st["q"].shape), lse


def _exact_router(st):
    """The losses and weights in 64 bits, their gradient by torch's differentiation with the counts held fixed."""
    c = st["case"]
    e, k, t = c["experts"], c["top_k"], c["tokens"]
    keep = (st["mask"] != 0) if st["mask"] is not None else torch.ones(t, dtype=torch.bool, device=DEV)
    z = st["logits"].double()[keep].requires_grad_()
    n = z.shape[0]
    logp = torch.log_softmax(z, -1)
    pick = torch.argsort(z.detach(), dim=-1, descending=True, stable=True)[:, :k]
    w = torch.gather(logp, 1, pick)
    w = torch.softmax(w, -1) if c["normalize"] else w.exp()
    count = torch.bincount(pick.reshape(-1), minlength=e)
    mean = logp.exp().sum(0) / max(n, 1)
    losses = torch.stack([BALANCE * e * (count.double() / max(n * k, 1) * mean).sum(),
                          ZLOSS * torch.logsumexp(z, -1).square().sum() / max(n, 1)])
    (dz,) = torch.autograd.grad((losses * st["dlosses"].double()).sum() + (w * st["dweights"][keep].double()).sum(), z)
    index = torch.full((t, k), -1, dtype=torch.int32, device=DEV)
    weights, dlogits = torch.zeros((t, k), dtype=torch.float64, device=DEV), torch.zeros((t, e), dtype=torch.float64, device=DEV)
    index[keep], weights[keep], dlogits[keep] = pick.to(torch.int32), w.detach(), dz
    return {"index": index, "weights": weights, "counts": torch.cat([count, torch.tensor([n], device=DEV)]).to(torch.int32),
            "mean": mean.detach(), "losses": losses.detach(), "dlogits": dlogits}
