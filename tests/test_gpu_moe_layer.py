"""The example's layer against the same layer in 64 bits under autograd.

The library rounds to bf16 where rows are stored: up, gate's pre-activation, hidden, out, y and their gradients, each a relative
2^-9 of that tensor; along the longest chain (y -> out -> hidden -> gate -> x) that is at most eight roundings, and the sums mix
independent errors: 8 * 2^-9 = 2^-6 of the tensor's norm bounds the error of each gradient in the 2-norm."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("T,H,N,E,K,R", [(64, 256, 128, 8, 2, 2), (200, 136, 72, 12, 3, 4), (8, 64, 64, 16, 4, 8)])
def test_layer_and_its_gradients(T, H, N, E, K, R):
    from moe_layer import MoELayer
    layer = MoELayer(T, H, N, E, K, R, coef=0.5)
    g = torch.Generator(device="cuda").manual_seed(1)
    x, dy = (torch.randn(T, H, generator=g, device="cuda").bfloat16() for _ in range(2))
    y = layer.forward(x)
    grads = layer.backward(dy, torch.full((1,), 2.0, device="cuda"))
    assert int(layer.lay.status) == 0 and int(layer.routing.status) == 0

    leaf = {k: getattr(layer, k).double().requires_grad_(True) for k in ("w_gate", "w_up", "w_down")}
    xd = x.double().requires_grad_(True)
    logits = xd @ layer.w_router.double().t()
    p = torch.softmax(logits, 1)
    idx = layer.routing.topk_idx.long()
    assert torch.equal(torch.sort(idx, 1).values, torch.sort(torch.topk(logits, K, dim=1).indices, 1).values)
    w = torch.gather(p, 1, idx)
    w = w / w.sum(1, keepdim=True)
    rows = [torch.zeros(T, H, dtype=torch.float64, device="cuda")]
    for k in range(K):
        wg, wu, wd = (leaf[n][idx[:, k]] for n in ("w_gate", "w_up", "w_down"))
        h = torch.nn.functional.silu(torch.einsum("tnh,th->tn", wg, xd)) * torch.einsum("tnh,th->tn", wu, xd)
        rows.append(w[:, k:k + 1] * torch.einsum("thn,tn->th", wd, h))
    out = sum(rows)
    counts = torch.bincount(idx.flatten(), minlength=E).double()
    loss = 0.5 * (counts * E / (T * K) * p.mean(0)).sum()
    assert abs(float(layer.routing.loss) - float(loss)) < 1e-5
    ((out * dy.double()).sum() + 2.0 * loss).backward()

    def close(got, want):
        return float((got.double() - want).norm() / want.norm()) < 2.0 ** -6

    assert close(y, out.detach()) and close(grads["x"], xd.grad)
    for name, t in leaf.items():
        assert close(grads[name], t.grad), name
