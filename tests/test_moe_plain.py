"""The 64-bit statements the GPU tests compare with, pinned by differences and closed forms (CPU)."""
import math

import pytest
import torch

import moe_plain as plain


def _difference(fn, at, direction, h=1e-5):
    return (fn(at + h * direction) - fn(at - h * direction)) / (2 * h)


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("renormalize", [False, True])
def test_router_gradient_against_differences(sigmoid, renormalize):
    g = torch.Generator().manual_seed(3)
    T, E, K = 7, 9, 3
    l = torch.randn(T, E, generator=g, dtype=torch.float64)
    l[2, 4] = -math.inf
    l[5] = -math.inf
    idx, _ = plain.route(l, K, sigmoid)
    dw = torch.randn(T, K, generator=g, dtype=torch.float64)
    got = plain.route_gradient(l, idx, dw, sigmoid, renormalize, 2.5, coef=0.3, d_loss=1.7)

    def objective(v):
        s, _ = plain.scores(v, sigmoid)
        p = torch.where(idx >= 0, torch.gather(s, 1, idx.clamp(min=0).long()), 0.0)
        w = 2.5 * (p / p.sum(1, keepdim=True).clamp(min=1e-300) if renormalize else p)
        return float((w * dw).sum() + 1.7 * plain.balance(v, idx, sigmoid, 0.3)[3])

    for seed in range(4):
        d = torch.randn(T, E, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)
        want = _difference(objective, l, torch.where(torch.isfinite(l), d, 0.0))
        assert abs(float((got * d).sum()) - want) < 1e-7 * max(1.0, abs(want))
    assert float(got[5].abs().max()) == 0 and float(got[2, 4]) == 0


def test_balance_loss_of_an_even_batch_is_its_coefficient():
    E, K = 8, 2
    idx = torch.tensor([[(K * t + k) % E for k in range(K)] for t in range(12)], dtype=torch.int32)
    counts, n, mean, loss = plain.balance(torch.zeros(12, E), idx, False, 0.25)
    assert counts.tolist() == [3] * E and n == 12
    assert float(mean.sum()) == pytest.approx(1.0) and float(loss) == pytest.approx(0.25)


@pytest.mark.parametrize("name", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("op", ["none", "add", "mul"])
def test_experts_gradient_against_differences(name, op):
    g = torch.Generator().manual_seed(5)
    offsets, E, H, N = torch.tensor([0, 3, 3, 8]), 3, 5, 4
    P = 8

    def mk(*shape):
        return torch.randn(*shape, generator=g, dtype=torch.float64)

    x, w, b, r, dy = mk(P, H), mk(E, N, H), mk(E, N), mk(P, N), mk(P, N)
    operand = None if op == "none" else r

    def objective(x_, w_, b_, r_):
        return float((plain.experts(x_, offsets, w_, b_, name, None if op == "none" else r_, op == "mul")[0] * dy).sum())

    z = plain.experts(x, offsets, w, b, name)[1]
    got, _ = plain.experts_gradient(dy, x, offsets, w, z, name, operand, op == "mul")
    for i, key in enumerate(["dx", "dweight", "dbias", "doperand"]):
        at = [x, w, b, r]
        d = mk(*at[i].shape)
        want = _difference(lambda v: objective(*[v if j == i else a for j, a in enumerate(at)]), at[i], d, 1e-6)
        have = got[key] if key != "doperand" or op == "mul" else (dy if op == "add" else torch.zeros_like(dy))
        assert abs(float((have * d).sum()) - want) < 1e-6 * max(1.0, abs(want)), key
