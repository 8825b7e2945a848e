"""Plain 64-bit statements of the norm, the sorted experts, their products and the clipped gradient, for the tests: no library
code.  With the results come the sums of absolute terms that bound what fp32 sums on the way cost."""
import math

import torch

F64 = torch.float64


def half_step(dtype):
    """Of a rounding to the type, relative."""
    return torch.finfo(dtype).eps / 2


def norm(h, w, eps):
    """(y, 1 / root mean square) of rows h, the weight or None."""
    h = h.double()
    r = 1.0 / torch.sqrt(h.square().mean(1, keepdim=True) + eps)
    return h * r * (1.0 if w is None else w.double()), r


def e4m3(y, block):
    """(scale, y / scale) of rows y: the values before they are rounded to 8 bits."""
    d = y.shape[1]
    step = block or d
    scale = torch.stack([(y[:, i:i + step].abs().amax(1) / 448.0).clamp(min=2.0 ** -126) for i in range(0, d, step)], 1)
    return scale, y / scale.repeat_interleave(step, 1)[:, :d]


def norm_gradient(h, dy, w, dt, eps):
    """(dx, its absolute terms, dw, its absolute terms) by the formula."""
    h, dy = h.double(), dy.double()
    w = torch.ones(h.shape[1], dtype=F64, device=h.device) if w is None else w.double()
    r = 1.0 / torch.sqrt(h.square().mean(1, keepdim=True) + eps)
    n, g = h * r, dy * w
    dx = r * (g - n * (g * n).mean(1, keepdim=True))
    terms = r * (g.abs() + n.abs() * (g * n).abs().mean(1, keepdim=True))
    if dt is not None:
        dx, terms = dx + dt.double(), terms + dt.double().abs()
    return dx, terms, (dy * n).sum(0), (dy * n).abs().sum(0)


def sort(index, experts):
    """(offsets, place), choice by choice."""
    flat = index.cpu().reshape(-1).tolist()
    count = [sum(1 for e in flat if e == x) for x in range(experts)] if experts <= 8 else torch.bincount(
        torch.tensor([e for e in flat if 0 <= e < experts], dtype=torch.int64), minlength=experts).tolist()
    first = [0]
    for n in count:
        first.append(first[-1] + n)
    at, place = list(first), []
    for e in flat:
        place.append(at[e] if 0 <= e < experts else -1)
        if 0 <= e < experts:
            at[e] += 1
    return torch.tensor(first, dtype=torch.int32), torch.tensor(place, dtype=torch.int32).view(index.shape)


def combine(rows, place, weight):
    """(y, its absolute terms)."""
    t, k = place.shape
    y = torch.zeros(t, rows.shape[1], dtype=F64, device=rows.device)
    terms = torch.zeros_like(y)
    for j in range(k):
        some = (place[:, j] >= 0) & (place[:, j] < rows.shape[0])
        part = rows[place[some, j].long()].double() * (1.0 if weight is None else weight[some, j:j + 1].double())
        y[some] += part
        terms[some] += part.abs()
    return y, terms


def combine_gradient(dy, rows, place, weight):
    """(drows, which rows it writes, dweight, its absolute terms)."""
    drows = torch.zeros(rows.shape, dtype=F64, device=rows.device)
    live = torch.zeros(rows.shape[0], dtype=torch.bool, device=rows.device)
    dw = torch.zeros(place.shape, dtype=F64, device=rows.device)
    terms = torch.zeros_like(dw)
    for j in range(place.shape[1]):
        some = (place[:, j] >= 0) & (place[:, j] < rows.shape[0])
        p, d = place[some, j].long(), dy[some].double()
        drows[p] = d * weight[some, j:j + 1].double()
        live[p] = True
        dw[some, j] = (d * rows[p].double()).sum(1)
        terms[some, j] = (d * rows[p].double()).abs().sum(1)
    return drows, live, dw, terms


def spans(offsets, rows):
    """(first, end) of every expert as the offsets are read: the largest so far, within the rows."""
    out, most = [], 0
    for o in (int(x) for x in offsets.cpu()):
        out.append(most)
        most = max(most, min(max(o, 0), rows))
        out[-1] = most
    return list(zip(out[:-1], out[1:]))


def product(x, w, offsets, transposed):
    """(y, its absolute terms, which rows it writes)."""
    y = torch.zeros(x.shape[0], w.shape[1 if transposed else 2], dtype=F64, device=x.device)
    terms, live = torch.zeros_like(y), torch.zeros(x.shape[0], dtype=torch.bool, device=x.device)
    for e, (a, b) in enumerate(spans(offsets, x.shape[0])):
        if b > a:
            m = w[e].double().T if transposed else w[e].double()
            y[a:b], terms[a:b], live[a:b] = x[a:b].double() @ m, x[a:b].double().abs() @ m.abs(), True
    return y, terms, live


def product_weights(x, y, offsets):
    """(dw, its absolute terms)."""
    dw = torch.zeros(len(offsets) - 1, x.shape[1], y.shape[1], dtype=F64, device=x.device)
    terms = torch.zeros_like(dw)
    for e, (a, b) in enumerate(spans(offsets, x.shape[0])):
        dw[e], terms[e] = x[a:b].double().T @ y[a:b].double(), x[a:b].double().abs().T @ y[a:b].double().abs()
    return dw, terms


def squares(gradients):
    return math.fsum(float(g.double().square().sum()) for g in gradients)
