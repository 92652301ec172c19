"""Plain 64-bit statements of the router, the balance loss and the experts' products (torch, CPU or GPU), written from the
formulas in `include/ep.h` and sharing nothing with the CUDA path."""
import math

import torch


# ------------------------------------------------------------------------------------------------------- router

def masked(logits):
    """Experts that may not be picked: -inf, NaN, +inf."""
    l = logits.double()
    return ~torch.isfinite(l)


def scores(logits, sigmoid):
    """(score, probability) per token and expert, 0 where masked."""
    l, dead = logits.double(), masked(logits)
    safe = torch.where(dead, 0.0, l)
    if sigmoid:
        s = torch.where(dead, 0.0, torch.sigmoid(safe))            # (written out, its derivative is inf * 0 for the lowest logits)
        total = s.sum(1, keepdim=True)
        return s, s / torch.where(total == 0, 1.0, total)
    top = torch.where(dead, -math.inf, l).amax(1, keepdim=True)
    e = torch.where(dead, 0.0, torch.exp(safe - torch.where(torch.isinf(top), 0.0, top)))
    total = e.sum(1, keepdim=True)
    p = e / torch.where(total == 0, 1.0, total)
    return p, p


def route(logits, K, sigmoid=False, bias=None, renormalize=True, scale=1.0, order_by=None):
    """order_by: the values the picks are ordered by, if not the 64-bit ones (a test that wants fp32's rounding of them)."""
    dead = masked(logits)
    s, _ = scores(logits, sigmoid)
    v = order_by if order_by is not None else (logits.double() if bias is None else s + bias.double())
    v = torch.where(dead, -math.inf, v.double())
    T, E = logits.shape
    order = torch.sort(v, dim=1, descending=True, stable=True)          # equal values stay in the order of their ids
    n = min(K, E)
    some = order.values[:, :n] > -math.inf
    idx = torch.full((T, K), -1, dtype=torch.int32)
    w = torch.zeros(T, K, dtype=torch.float64)
    idx[:, :n] = torch.where(some, order.indices[:, :n], -1).to(torch.int32)
    picked = torch.where(some, torch.gather(s, 1, order.indices[:, :n]), 0.0)
    total = picked.sum(1, keepdim=True) if renormalize else torch.ones(T, 1, dtype=torch.float64)
    w[:, :n] = torch.where(total > 0, scale * picked / torch.where(total > 0, total, 1.0), 0.0)
    return idx, w


def balance(logits, topk_idx, sigmoid, coef):
    """(counts, tokens, mean probabilities, loss); differentiable in the logits."""
    T, E = logits.shape
    _, p = scores(logits, sigmoid)
    ok = (topk_idx >= 0) & (topk_idx < E)
    counts = torch.bincount(topk_idx[ok].long(), minlength=E)
    token = ok.any(1) & ~masked(logits).all(1)
    n = int(token.sum())
    mean = (p * token[:, None]).sum(0) / max(1, n)
    f = counts.double() * E / max(1, int(counts.sum()))
    return counts.to(torch.int32), n, mean, coef * (f * mean).sum()


def route_gradient(logits, topk_idx, d_weights, sigmoid, renormalize, scale, coef=0.0, d_loss=0.0):
    """Gradient of sum(d_weights * weights) + d_loss * loss with respect to the logits, by differentiating the 64-bit forms."""
    dead = masked(logits)
    l = torch.where(dead, -math.inf, logits.double()).requires_grad_(True)
    s, _ = scores(l, sigmoid)
    ok = topk_idx >= 0
    picked = torch.where(ok, torch.gather(s, 1, topk_idx.clamp(min=0).long()), 0.0)
    total = picked.sum(1, keepdim=True)
    w = scale * (picked / torch.where(total == 0, 1.0, total) if renormalize else picked)
    objective = (w * d_weights.double()).sum() if d_weights is not None else 0.0
    if coef:
        objective = objective + d_loss * balance(l, topk_idx, sigmoid, coef)[3]
    g, = torch.autograd.grad(objective, l)
    return torch.where(dead | ~ok.any(1, keepdim=True), 0.0, g)


# ------------------------------------------------------------------------------------------------------ experts

def act(z, name):
    return {"none": lambda v: v, "relu": torch.relu, "silu": lambda v: v / (1 + torch.exp(-v)),
            "gelu": lambda v: 0.5 * v * (1 + torch.erf(v * math.sqrt(0.5)))}[name](z)


def slope(z, name):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s + z * s * (1 - s)
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return torch.ones_like(z)


def segments(offsets):
    o = [int(v) for v in offsets]
    return [slice(o[e], o[e + 1]) for e in range(len(o) - 1)]


def experts(x, offsets, weight, bias=None, name="none", operand=None, mul=False):
    """(y, z, S): the result, what the activation is applied to, and the sums of absolute products that bound z's error."""
    P = int(offsets[-1])
    E, N, H = weight.shape
    z = torch.zeros(P, N, dtype=torch.float64, device=x.device)
    S = torch.zeros_like(z)
    for e, rows in enumerate(segments(offsets)):
        xe, we = x[rows].double(), weight[e].double()
        z[rows] = xe @ we.t() + (0 if bias is None else bias[e].double())
        S[rows] = xe.abs() @ we.abs().t() + (0 if bias is None else bias[e].double().abs())
    y = act(z, name)
    if operand is not None:
        y = y * operand[:P].double() if mul else y + operand[:P].double()
    return y, z, S


def experts_gradient(dy, x, offsets, weight, pre, name="none", operand=None, mul=False):
    """dx, dweight, dbias, doperand and, for the error bounds, the same sums over absolute values (all 64 bits); size["slope"] is
    what an error of 1 in the slope of every row would do to dbias, weighted with 1 + |z|."""
    P = int(offsets[-1])
    E, N, H = weight.shape
    g = dy[:P].double()
    z = pre[:P].double() if pre is not None else torch.zeros_like(g)
    dop = g * act(z, name) if mul else None
    if mul:
        g = g * operand[:P].double()
    dz = g * slope(z, name)
    out = {"dx": torch.zeros(P, H, dtype=torch.float64, device=dy.device),
           "dweight": torch.zeros(E, N, H, dtype=torch.float64, device=dy.device),
           "dbias": torch.zeros(E, N, dtype=torch.float64, device=dy.device), "doperand": dop}
    size = {k: torch.zeros_like(v) for k, v in out.items() if k != "doperand"}
    size["slope"] = torch.zeros_like(out["dbias"])
    for e, rows in enumerate(segments(offsets)):
        xe, we, de = x[rows].double(), weight[e].double(), dz[rows]
        out["dx"][rows], size["dx"][rows] = de @ we, de.abs() @ we.abs()
        out["dweight"][e], size["dweight"][e] = de.t() @ xe, de.t().abs() @ xe.abs()
        out["dbias"][e], size["dbias"][e] = de.sum(0), de.abs().sum(0)
        size["slope"][e] = (g[rows].abs() * (1 + z[rows].abs())).sum(0)
    return out, size
