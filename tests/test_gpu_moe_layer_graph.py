"""The example's layer in a CUDA graph: a step captured once and replayed on other inputs, masked tokens among them."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_a_training_step_replays_from_a_graph():
    from moe_layer import MoELayer
    T, H, N, E, K, R = 64, 256, 128, 8, 2, 2
    layer, d_loss = MoELayer(T, H, N, E, K, R, coef=0.5), torch.full((1,), 2.0, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(3)
    inputs = [[torch.randn(T, H, generator=g, device="cuda").bfloat16() for _ in range(2)] for _ in range(3)]
    inputs[2][0][7] = float("nan")                              # a token whose logits are all NaN has no pick, and one pair less each
    want = []
    for x, dy in inputs:
        y = layer.forward(x).clone()
        want.append((y, {k: v.clone() for k, v in layer.backward(dy, d_loss).items()}))
    x, dy = (t.clone() for t in inputs[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                               # torch's products set their handles up outside the capture
        layer.forward(x), layer.backward(dy, d_loss)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = layer.forward(x)
        grads = layer.backward(dy, d_loss)
    for (xi, dyi), (yi, gi) in zip(inputs, want):
        x.copy_(xi), dy.copy_(dyi)
        graph.replay()
        assert torch.equal(y, yi)
        for k in gi:
            assert torch.equal(grads[k], gi[k]) or (k == "x" and torch.equal(torch.isnan(grads[k]), torch.isnan(gi[k]))), k
    assert int(layer.lay.status) == 0 and (want[2][0][7] == 0).all()
