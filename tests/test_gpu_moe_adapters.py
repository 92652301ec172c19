"""The fine-tuning example: the sort, the adapters, dropout and the combine together, against the same layer in 64 bits under autograd.

The library rounds to bf16 where rows are stored; along the longest chain (y -> d_out -> d_hidden -> d_up -> dmid -> ddown, and x -> up ->
hidden -> mid -> out on the way there) these are at most ten roundings of 2^-9 relative to a tensor's norm, on average half of that, and they mix in sums:
10 * 2^-9 bounds the error of each gradient in the 2-norm."""
import os
import sys

import pytest
import torch

import train_plain as plain

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def _reference(layer, x, dy, step):
    """y and the gradients, for the picks and the masks that the layer has."""
    T, H, E, K = layer.T, layer.H, layer.E, layer.K
    slot, idx = layer.lay.pair_slot.long().cpu(), layer.routing.topk_idx.long().cpu()
    live = slot >= 0
    seed, p = int(layer.random[0]), layer.drop_x.p
    leaf = {"x": x, "up_down": layer.on_up.down, "up_up": layer.on_up.up, "down_down": layer.on_down.down, "down_up": layer.on_down.up,
            "topk_weights": layer.routing.topk_weights}
    leaf = {k: v.double().cpu().requires_grad_(True) for k, v in leaf.items()}
    wg, wu, wd, s = (t.double().cpu() for t in (layer.w_gate, layer.w_up, layer.w_down, layer.on_up.scale))
    keep_x, keep_y = plain.keep(layer.P, H, p, seed, step, 0), plain.keep(T, H, p, seed, step, 1)
    acc = [torch.zeros(T, H, dtype=torch.float64)]
    for k in range(K):
        t = torch.nonzero(live[:, k]).flatten()
        e, row = idx[t, k], leaf["x"][t]
        xd = row * keep_x[slot[t, k]]
        mv = lambda w, v: torch.einsum("tab,tb->ta", w, v)                   # noqa: E731
        up = mv(wu[e], row) + s[e, None] * mv(leaf["up_up"][e], mv(leaf["up_down"][e], xd))
        hidden = torch.nn.functional.silu(mv(wg[e], row)) * up
        out = mv(wd[e], hidden) + s[e, None] * mv(leaf["down_up"][e], mv(leaf["down_down"][e], hidden))
        acc.append(torch.zeros(T, H, dtype=torch.float64).index_add(0, t, leaf["topk_weights"][t, k, None] * out))
    y = leaf["x"] + sum(acc) * keep_y
    (y * dy.double().cpu()).sum().backward()
    return y.detach(), {k: v.grad for k, v in leaf.items()}


def _close(got, want, name):
    err = float((got.double().cpu() - want).norm() / want.norm().clamp(min=1e-30))
    assert err < 10 * 2.0 ** -9, (name, err)


@pytest.mark.parametrize("T,H,N,E,K,rank,p", [(64, 256, 128, 8, 2, 16, 0.25), (50, 136, 72, 12, 3, 8, 0.0), (9, 64, 64, 16, 4, 24, 0.5)])
def test_layer_and_its_gradients(T, H, N, E, K, rank, p):
    from moe_adapters import AdaptedMoE
    layer = AdaptedMoE(T, H, N, E, K, rank, p=p, scale=2.0 * rank)
    g = torch.Generator(device="cuda").manual_seed(1)
    x, dy = (torch.randn(T, H, generator=g, device="cuda").bfloat16() for _ in range(2))
    for step in range(2):
        y, grads = layer.step(x, dy)
        assert int(layer.lay.status) == 0 and int(layer.routing.status) == 0
        want, wanted = _reference(layer, x, dy, step)
        _close(y, want, "y")
        for name, t in wanted.items():
            _close(grads[name], t, name)


def test_a_step_replays_from_a_graph_with_new_masks():
    from moe_adapters import AdaptedMoE
    T, H, N, E, K, rank = 64, 128, 64, 8, 2, 16
    g = torch.Generator(device="cuda").manual_seed(3)
    inputs = [[torch.randn(T, H, generator=g, device="cuda").bfloat16() for _ in range(2)] for _ in range(3)]
    inputs[2][0][7] = float("nan")                              # a token without a pick
    layer = AdaptedMoE(T, H, N, E, K, rank, p=0.3)
    want = []
    for x, dy in inputs:
        y, grads = layer.step(x, dy)
        want.append((y.clone(), {k: v.clone() for k, v in grads.items()}))
    layer.random[1] = 0
    x, dy = (t.clone() for t in inputs[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                               # torch's product sets its handle up outside the capture
        layer.forward(x)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, grads = layer.step(x, dy)
    for (xi, dyi), (yi, gi) in zip(inputs, want):
        x.copy_(xi), dy.copy_(dyi)
        graph.replay()
        assert torch.equal(y.view(torch.int16), yi.view(torch.int16))
        for k in gi:
            assert torch.equal(torch.nan_to_num(grads[k].float(), 7.0), torch.nan_to_num(gi[k].float(), 7.0)), k
    assert int(layer.lay.status) == 0
