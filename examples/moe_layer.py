"""One mixture-of-experts layer, forward and backward, on the library's calls:

    router -> layout + dispatch -> group -> gated experts -> combine        y = sum_k w_k W2_e( silu(Wg_e x) * (Wu_e x) )

with the balance loss, and the gradients of the input, the router's logits and the experts' weights. The router's projection, the
gradient of the combine's weights and the sum of the two branches' gradients are torch, and part of the times. Nothing waits for the GPU,
so that a step can be captured in a CUDA graph.

    python examples/moe_layer.py [--tokens 4096 --hidden 2048 --inner 1024 --experts 128 --top-k 8 --ranks 8 --steps 10]

prints the time of a training step and of the forward pass alone (random weights and inputs).
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2609_40093_b200 import ep  # noqa: E402


class MoELayer:
    """Weights, and the buffers of one batch size. The R expert-parallel ranks are partitions of this GPU's buffers."""

    def __init__(self, T, H, N, E, K, R, coef=0.01, seed=0, device="cuda"):
        self.T, self.H, self.N, self.E, self.K, self.R = T, H, N, E, K, R
        g = torch.Generator(device=device).manual_seed(seed)

        def weight(*shape):
            return (torch.randn(*shape, generator=g, device=device) * shape[-1] ** -0.5).bfloat16()

        self.w_router = torch.randn(E, H, generator=g, device=device) * H ** -0.5
        self.w_gate, self.w_up, self.w_down = weight(E, N, H), weight(E, N, H), weight(E, H, N)
        self.router = ep.Router(E, K, balance_coef=coef)
        P = T * K

        def rows(n, cols):
            return torch.empty(n, cols, dtype=torch.bfloat16, device=device)

        self.routing = ep.alloc_routing(T, E, K, balance=True, device=device)
        self.lay = ep.alloc_layout(T, K, E, R, device=device, fill=-1)      # -1: rows behind the last pair name no token
        self.ws = torch.empty(max(16, ep.ep_layout_workspace_bytes(T, K, E, R)), dtype=torch.uint8, device=device)
        self.recv, self.x, self.up, self.gate = rows(T * min(K, R), H), rows(P, H), rows(P, N), rows(P, N)
        self.hidden, self.out, self.y = rows(P, N), rows(P, H), rows(T, H)
        self.ones = torch.ones(T, K, device=device)

    def forward(self, x):
        """x [T, H] bf16 -> y [T, H] bf16; the loss is in self.routing.loss."""
        E, R, lay, r = self.E, self.R, self.lay, self.routing
        self.logits = x.float() @ self.w_router.t()
        ep.ep_route(self.logits, self.router, out=r)
        ep.ep_layout_dispatch(r.topk_idx, x, self.recv, E, R, lay, self.ws)
        ep.ep_group(self.recv, lay, self.x, E, R, status=lay.status)
        off = lay.expert_offsets
        ep.ep_expert_matmul(self.x, off, self.w_up, y=self.up, status=lay.status)
        ep.ep_expert_matmul(self.x, off, self.w_gate, activation=ep.ACT_SILU, operand=self.up, operand_op=ep.OPERAND_MUL, y=self.hidden,
                            pre=self.gate, status=lay.status)
        ep.ep_expert_matmul(self.hidden, off, self.w_down, y=self.out, status=lay.status)
        return ep.ep_combine(self.out, lay.pair_slot, r.topk_weights, self.y, E, R, status=lay.status)

    def backward(self, dy, d_loss):
        """Gradients of sum(dy * y) + d_loss * loss: a dict of tensors."""
        T, H, N, E, K, R, lay, r = self.T, self.H, self.N, self.E, self.K, self.R, self.lay, self.routing
        P, off = T * K, lay.expert_offsets
        slot = lay.pair_slot.long().clamp(min=0)
        valid = lay.pair_slot >= 0
        # combine: a pair's output row gets its token's gradient times its weight, its weight the product of the two rows
        w_pair = torch.zeros(P + 1, 1, device=dy.device)                    # entries that name no pair go to the last one
        w_pair[torch.where(valid, slot, P), 0] = r.topk_weights
        d_out = ep.ep_combine(dy, lay.pair_token.view(P, 1), w_pair[:P], torch.empty(P, H, dtype=torch.bfloat16, device=dy.device), 1, 1)
        d_weights = torch.stack([(dy.float() * self.out[slot[:, k]].float()).sum(1) for k in range(K)], 1) * valid
        down = ep.ep_expert_matmul_backward(d_out, self.hidden, off, self.w_down, status=lay.status)
        gate = ep.ep_expert_matmul_backward(down.dx, self.x, off, self.w_gate, pre=self.gate, activation=ep.ACT_SILU, operand=self.up,
                                            operand_op=ep.OPERAND_MUL, grads=ep.alloc_expert_grads(P, H, N, E, operand=True), status=lay.status)
        up = ep.ep_expert_matmul_backward(gate.doperand, self.x, off, self.w_up, status=lay.status)
        # dispatch: a token's rows come back with unit weights, here from the pair space, once per branch
        dx = torch.empty_like(dy)
        ep.ep_combine(gate.dx, lay.pair_slot, self.ones, dx, E, R)
        dx = dx + ep.ep_combine(up.dx, lay.pair_slot, self.ones, torch.empty_like(dy), E, R)
        d_logits = ep.ep_route_backward(self.logits, self.router, r, d_weights=d_weights, d_loss=d_loss)
        return {"x": dx.float() + d_logits @ self.w_router, "w_gate": gate.dweight, "w_up": up.dweight, "w_down": down.dweight,
                "logits": d_logits, "topk_weights": d_weights}


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, default in (("tokens", 4096), ("hidden", 2048), ("inner", 1024), ("experts", 128), ("top-k", 8), ("ranks", 8), ("steps", 10)):
        ap.add_argument("--" + name, type=int, default=default)
    a = ap.parse_args()
    layer = MoELayer(a.tokens, a.hidden, a.inner, a.experts, a.top_k, a.ranks)
    x, dy = (torch.randn(a.tokens, a.hidden, device="cuda").bfloat16() for _ in range(2))
    d_loss = torch.ones(1, device="cuda")

    def timed(fn):
        for _ in range(3):
            fn()
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        torch.cuda.synchronize()
        begin.record()
        for _ in range(a.steps):
            fn()
        end.record()
        torch.cuda.synchronize()
        return begin.elapsed_time(end) / a.steps

    forward = timed(lambda: layer.forward(x))
    step = timed(lambda: (layer.forward(x), layer.backward(dy, d_loss)))
    status = ep.ep_status(layer.lay.status) | ep.ep_status(layer.routing.status)
    print(f"forward {forward:.3f} ms, forward and backward {step:.3f} ms, balance loss {float(layer.routing.loss):.5f}, "
          f"most loaded expert {int(layer.routing.expert_counts.max())} of {a.tokens * a.top_k} pairs, status {status}")


if __name__ == "__main__":
    main()
