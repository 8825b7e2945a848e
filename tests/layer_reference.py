"""Plain 64-bit statements of the decoder-layer operators, for the tests: loops over samples and heads, no library code.

Each also gives, where outputs are rounded to 16 bits on the way, the sums of absolute terms that bound what that costs."""
import math

import torch

U = 2.0 ** -8                 # half a unit in the last place of bfloat16, relative


def rotary_table(positions, r, base=10000.0, scaling="plain", factor=1.0, trained=4096.0, slow=1.0, fast=32.0, magnitude=1.0):
    j = torch.arange(r // 2, dtype=torch.float64)
    w = base ** (-2.0 * j / r)
    if scaling == "linear":
        w = w / factor
    elif scaling == "parts":
        keep = ((trained * w / (2 * math.pi) - slow) / (fast - slow)).clamp(0, 1)
        w = w / factor * (1 - keep) + w * keep
    a = torch.arange(positions, dtype=torch.float64)[:, None] * w
    return torch.cat([a.cos(), a.sin()], 1) * magnitude


def rotary(x, table, positions, layout, inverse):
    """x [batch, seq, heads, dim]; positions [batch, seq]."""
    x, r = x.double().cpu(), table.shape[1]
    h = r // 2
    t = table.double().cpu()[positions.cpu().long()][:, :, None]
    c, s = t[..., :h], t[..., h:] * (-1 if inverse else 1)
    y = x.clone()
    for j in range(h):
        a, b = (j, j + h) if layout == "half" else (2 * j, 2 * j + 1)
        y[..., a] = x[..., a] * c[..., j] - x[..., b] * s[..., j]
        y[..., b] = x[..., b] * c[..., j] + x[..., a] * s[..., j]
    return y


def _seen(nq, nk, causal, device):
    see = torch.ones(nq, nk, dtype=torch.bool, device=device)
    return see.tril(nk - nq) if causal else see


def attention(q, k, v, causal, scale):
    """One sample and head, [rows, dim]: (o, lse, sum of p |v|)."""
    q, k, v = q.double(), k.double(), v.double()
    if k.shape[0] == 0:
        return torch.zeros_like(q), torch.full((q.shape[0],), -math.inf, dtype=torch.float64, device=q.device), torch.zeros_like(q)
    s = (q @ k.T * scale).masked_fill(~_seen(len(q), len(k), causal, q.device), -math.inf)
    lse = torch.logsumexp(s, 1)
    p = torch.where(lse[:, None] > -math.inf, torch.exp(s - torch.where(lse > -math.inf, lse, 0.0)[:, None]), 0.0)
    return p @ v, lse, p @ v.abs()


def attention_gradient(q, k, v, o, lse, do, causal, scale):
    """One sample and head: (dq, dk, dv) by the formula with the given o and lse, and their sums of absolute terms."""
    q, k, v, o, lse, do = (t.double() for t in (q, k, v, o, lse, do))
    see = _seen(len(q), len(k), causal, q.device)
    p = torch.where(see & (lse[:, None] > -math.inf), torch.exp(q @ k.T * scale - torch.where(lse > -math.inf, lse, 0.0)[:, None]), 0.0)
    dp, dot = do @ v.T, (do * o).sum(1, keepdim=True)
    ds = p * (dp - dot)
    return (ds @ k * scale, ds.T @ q * scale, p.T @ do,
            ds.abs() @ k.abs() * abs(scale), ds.abs().T @ q.abs() * abs(scale), p.T @ do.abs())


def router(z, k, normalize, balance, zcoef, mask=None):
    """(index, weight, counts, mean, losses) of fp64 logits that may require a gradient."""
    n, e = z.shape
    index = torch.full((n, k), -1, dtype=torch.int32)
    counts = torch.zeros(e + 1, dtype=torch.int32)
    weight, mean, zsq = [], torch.zeros(e, dtype=torch.float64), torch.zeros((), dtype=torch.float64)
    for t in range(n):
        row = torch.zeros(k, dtype=torch.float64)
        free = [i for i in range(e) if float(z[t, i].detach()) != -math.inf]
        if free and (mask is None or int(mask[t])):
            counts[e] += 1
            lse = torch.logsumexp(z[t, free], 0)
            p = torch.exp(z[t] - lse)
            mean = mean + p
            zsq = zsq + lse * lse
            order = sorted(free, key=lambda i: (-float(z[t, i].detach()), i))[:k]
            share = sum(p[i] for i in order) if normalize else torch.ones((), dtype=torch.float64)
            parts = [p[i] / share for i in order] + [torch.zeros((), dtype=torch.float64)] * (k - len(order))
            row = torch.stack(parts)
            for j, i in enumerate(order):
                index[t, j] = i
                counts[i] += 1
        weight.append(row)
    act = max(int(counts[e]), 1)
    mean = mean / act
    losses = torch.stack([balance * e * (counts[:e].double() / (act * k) * mean).sum(), zcoef * zsq / act])
    return index, torch.stack(weight) if weight else torch.zeros(0, k, dtype=torch.float64), counts, mean, losses
