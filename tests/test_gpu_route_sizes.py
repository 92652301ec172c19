"""Router sizes between and beyond those of `test_gpu_route`: 513 to 768 experts, where a lane holds 24 values, and the ends of the
groups next to them. The tolerances are those of `test_gpu_route`."""
import math

import pytest
import torch

import moe_plain as plain
from paper_2609_40093_b200 import ep
from test_gpu_route import _compare_balance, _compare_route, _logits
from test_gpu_route_low_scores import _compare_gradient

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,E,K", [(9, 260, 8), (20, 384, 6), (8, 513, 3), (33, 600, 8), (7, 619, 9), (40, 768, 12), (5, 769, 4), (1, 640, 32), (300, 576, 8)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sigmoid", [False, True])
def test_many_values_a_lane(T, E, K, dtype, sigmoid):
    """Picks, weights, loss and gradients, with masked tokens and experts, NaN and equal logits."""
    logits = _logits(T, E, torch.float32, T + E)
    logits[::3] = (logits[::3] * 2).round() / 2                 # equal logits in a row
    logits[T // 2, ::2] = -math.inf
    if T > 4:
        logits[3] = -math.inf
        logits[4, E - 1] = math.nan
    logits = logits.to(dtype)
    for renormalize in (True, False):
        router = ep.Router(E, K, scoring=int(sigmoid), renormalize=renormalize, scale=1.5, balance_coef=0.4)
        _compare_route(logits, ep.Router(E, K, scoring=int(sigmoid), renormalize=renormalize, scale=1.5))
        got, idx = _compare_route(logits, router)
        assert int(got.status) == (ep.STATUS_BAD_LOGIT if T > 4 else 0)
        _compare_balance(got, logits, idx, sigmoid, 0.4)
        _compare_balance(ep.ep_balance_loss(logits.cuda(), router, idx.cuda()), logits, idx, sigmoid, 0.4)
        dw, dl = torch.randn(T, K, generator=torch.Generator().manual_seed(1)), 30.0
        grad = ep.ep_route_backward(logits.cuda(), router, got, d_weights=dw.cuda(), d_loss=torch.full((1,), dl, device="cuda"))
        _compare_gradient(grad, logits, idx, dw, sigmoid, renormalize, 1.5, 0.4, dl, int(got.tokens), got.expert_counts.cpu().double())
        bias = torch.randperm(E, generator=torch.Generator().manual_seed(2)).float() * 2         # orders alone
        biased = ep.ep_route(logits.cuda(), router, bias=bias.cuda(), out=ep.alloc_routing(T, E, K, balance=True))
        want, w = plain.route(logits, K, sigmoid, bias, renormalize, 1.5)
        assert torch.equal(biased.topk_idx.cpu(), want)
        assert ((biased.topk_weights.cpu().double() - w).abs() <= 2.0 ** -15 * w + 1e-7).all()
        _compare_balance(biased, logits, want, sigmoid, 0.4)
