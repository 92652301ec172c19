"""Fine-tuning a mixture-of-experts layer whose weights are frozen: every expert has a low-rank adapter beside its up and its down projection.

    y = x + drop( sum_k w_k out_e(x) )        up = Wu_e x + s Bu_e Au_e drop(x)     hidden = silu(Wg_e x) * up     out = Wd_e hidden + s Bd_e Ad_e hidden

Rows go to the pair space and back by ep_sort, ep_combine_residual and their gradients; the adapters' gradients are what a step trains. Dropout
takes its bits from a seed and a step on the device: the backward pass makes the same masks again, and a step captured in a CUDA graph takes new ones
at each replay, because it ends by counting the step up.

    python examples/moe_adapters.py [--tokens 4096 --hidden 2048 --inner 1024 --experts 128 --top-k 8 --rank 32 --p 0.1 --steps 10]

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


class AdaptedMoE:
    """Frozen weights, adapters, and the buffers of one batch size."""

    def __init__(self, T, H, N, E, K, rank, p=0.1, scale=2.0, seed=0, device="cuda"):
        self.T, self.H, self.N, self.E, self.K, self.P = T, H, N, E, K, T * K
        g = torch.Generator(device=device).manual_seed(seed)

        def weight(*shape):
            return (torch.randn(*shape, generator=g, device=device) * shape[-1] ** -0.5).bfloat16()

        self.w_router = torch.randn(E, H, generator=g, device=device) * H ** -0.5
        self.w_gate, self.w_up, self.w_down = weight(E, N, H), weight(E, N, H), weight(E, H, N)
        scales = torch.full((E,), scale / rank, device=device)
        self.on_up = ep.Adapters(weight(E, rank, H), weight(E, N, rank), scales)
        self.on_down = ep.Adapters(weight(E, rank, N), weight(E, H, rank), scales)
        self.random = torch.tensor([seed, 0], dtype=torch.int64, device=device)      # seed and step
        self.drop_x, self.drop_y = ep.Dropout(p, self.random, site=0), ep.Dropout(p, self.random, site=1)
        self.router = ep.Router(E, K)
        self.routing = ep.alloc_routing(T, E, K, device=device)
        self.lay = ep.alloc_layout(T, K, E, 1, device=device, fill=-1)
        self.ws = torch.empty(max(16, ep.ep_layout_workspace_bytes(T, K, E, 1)), dtype=torch.uint8, device=device)

        def rows(n, cols):
            return torch.zeros(n, cols, dtype=torch.bfloat16, device=device)

        P = self.P
        self.x, self.xd, self.up, self.gate, self.hidden, self.out = rows(P, H), rows(P, H), rows(P, N), rows(P, N), rows(P, N), rows(P, H)
        self.mid_up, self.mid_down, self.y = rows(P, rank), rows(P, rank), rows(T, H)
        self.d_out, self.d_hidden, self.dx_pairs, self.dx = rows(P, H), rows(P, N), rows(P, H), rows(T, H)
        self.d_weights = torch.zeros(T, K, device=device)
        self.g_up, self.g_down = ep.alloc_adapter_grads(self.xd, self.on_up), ep.alloc_adapter_grads(self.hidden, self.on_down)
        self.g_gate = ep.alloc_expert_grads(P, H, N, E, weight=False, operand=True, device=device)
        self.g_frozen = [ep.alloc_expert_grads(P, a, b, E, weight=False, device=device) for a, b in ((H, N), (N, H))]

    def forward(self, x):
        """x [T, H] bf16 -> y [T, H] bf16."""
        lay, st = self.lay, self.lay.status
        ep.ep_route(x.float() @ self.w_router.t(), self.router, out=self.routing)
        ep.ep_layout(self.routing.topk_idx, self.E, 1, out=lay, workspace=self.ws)
        ep.ep_sort(x, lay.pair_slot, self.x, status=st)
        off, pairs = lay.expert_offsets, lay.expert_offsets[self.E:]
        ep.ep_dropout(self.x, self.drop_x, y=self.xd, limit=pairs)
        ep.ep_expert_matmul(self.x, off, self.w_up, y=self.up, status=st)
        ep.ep_adapter_matmul(self.xd, off, self.on_up, self.up, base=self.up, mid=self.mid_up, status=st)
        ep.ep_expert_matmul(self.x, off, self.w_gate, activation=ep.ACT_SILU, operand=self.up, operand_op=ep.OPERAND_MUL, y=self.hidden,
                            pre=self.gate, status=st)
        ep.ep_expert_matmul(self.hidden, off, self.w_down, y=self.out, status=st)
        ep.ep_adapter_matmul(self.hidden, off, self.on_down, self.out, base=self.out, mid=self.mid_down, status=st)
        return ep.ep_combine_residual(self.out, lay.pair_slot, self.routing.topk_weights, self.y, residual=x, dropout=self.drop_y, status=st)

    def backward(self, dy):
        """Gradients of sum(dy * y): a dict of tensors (the adapters', the input's through the experts, the weights of the picks)."""
        lay, st, slot, off = self.lay, self.lay.status, self.lay.pair_slot, self.lay.expert_offsets
        pairs = off[self.E:]
        ep.ep_combine_backward(dy, slot, self.routing.topk_weights, self.d_out, out=self.out, d_weights=self.d_weights, dropout=self.drop_y, status=st)
        ep.ep_expert_matmul_backward(self.d_out, self.hidden, off, self.w_down, grads=self.g_frozen[1], status=st)
        self.g_down.dx = self.g_frozen[1].dx                                    # the adapter's share is added in place
        ep.ep_adapter_matmul_backward(self.d_out, self.hidden, off, self.on_down, self.mid_down, self.g_down, base=self.g_down.dx, status=st)
        gate = ep.ep_expert_matmul_backward(self.g_down.dx, self.x, off, self.w_gate, pre=self.gate, activation=ep.ACT_SILU, operand=self.up,
                                            operand_op=ep.OPERAND_MUL, grads=self.g_gate, status=st)
        d_up = gate.doperand
        ep.ep_expert_matmul_backward(d_up, self.x, off, self.w_up, grads=self.g_frozen[0], status=st)
        ep.ep_adapter_matmul_backward(d_up, self.xd, off, self.on_up, self.mid_up, self.g_up, status=st)
        # the adapter saw drop(x): its gradient goes through the same mask, onto the frozen projection's
        ep.ep_dropout(self.g_up.dx, self.drop_x, residual=self.g_frozen[0].dx, y=self.dx_pairs, limit=pairs)
        ep.ep_sort_backward(self.dx_pairs, slot, self.dx, add=dy, status=st)    # dy: the residual's gradient
        ep.ep_sort_backward(gate.dx, slot, self.dx, add=self.dx, status=st)
        return {"x": self.dx, "topk_weights": self.d_weights, "up_down": self.g_up.ddown, "up_up": self.g_up.dup, "down_down": self.g_down.ddown,
                "down_up": self.g_down.dup}

    def step(self, x, dy):
        y = self.forward(x)
        grads = self.backward(dy)
        self.random[1] += 1
        return y, grads


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, default in (("tokens", 4096), ("hidden", 2048), ("inner", 1024), ("experts", 128), ("top-k", 8), ("rank", 32), ("steps", 10)):
        ap.add_argument("--" + name, type=int, default=default)
    ap.add_argument("--p", type=float, default=0.1)
    a = ap.parse_args()
    layer = AdaptedMoE(a.tokens, a.hidden, a.inner, a.experts, a.top_k, a.rank, p=a.p)
    x, dy = (torch.randn(a.tokens, a.hidden, device="cuda").bfloat16() for _ in range(2))

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

    forward, step = timed(lambda: layer.forward(x)), timed(lambda: layer.step(x, dy))
    print(f"forward {forward:.3f} ms, forward and backward {step:.3f} ms, status {ep.ep_status(layer.lay.status)}")


if __name__ == "__main__":
    main()
