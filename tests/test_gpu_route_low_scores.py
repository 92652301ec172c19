"""Router, balance loss and gradients where the picked scores are so small that their sum, or its reciprocal, leaves fp32's normal
range: sigmoids of logits below -80, and picks that a selection bias takes from far below the largest logit of a softmax.

The tolerances of `test_gpu_route` hold there as well: the renormalised weights, the probabilities of the loss and their gradients
depend on differences of logits alone, which fp32 holds to 2^-24 of the logits (at most 104 here: 2^-17, below half of WEIGHT)."""
import pytest
import torch

import moe_plain as plain
from paper_2609_40093_b200 import ep
from test_gpu_route import TINY, WEIGHT, _compare_balance

pytestmark = pytest.mark.gpu

LEVELS = (-60.0, -79.0, -86.0, -88.0, -91.0, -95.0, -100.0, -102.0)
# a warp per token at one, two, four, ... values a lane, and a thread per token
SIZES = [(40, 8, 3), (40, 24, 4), (40, 60, 6), (24, 256, 8), (24, 300, 5), (16, 1030, 4), (16384, 8, 2), (32768, 16, 4)]


def _low_rows(T, E, seed, dtype=torch.float32):
    """Every other token's logits lie around one of LEVELS, half of 1 apart from each other."""
    g = torch.Generator().manual_seed(seed)
    logits = 1.5 * torch.randn(T, E, generator=g)
    low = torch.tensor(LEVELS)[torch.arange(T) // 2 % len(LEVELS)]
    logits[::2] = (low[:, None] + 0.5 * torch.rand(T, E, generator=g))[::2]
    if T > 21:
        logits[20] = -1.0e5                                     # scores of 0 in any precision
    return logits.to(dtype)


def _compare_gradient(got, logits, idx, dw, sigmoid, renormalize, scale, coef=0.0, d_loss=0.0, tokens=1, counts=None):
    want = plain.route_gradient(logits, idx, dw, sigmoid, renormalize, scale, coef, d_loss)
    s = plain.scores(logits, sigmoid)[0]
    picked = torch.where(idx >= 0, torch.gather(s, 1, idx.clamp(min=0).long()), 0.0)
    total = picked.sum(1, keepdim=True)
    unit = scale / torch.where(total > 0, total, 1.0) if renormalize else scale
    tol = 2.0 ** -14 * (dw.double().abs() * unit * picked).amax(1, keepdim=True) + 1e-30 if dw is not None else torch.zeros(1, 1) + 1e-30
    if coef:
        tol = tol + 2.0 ** -14 * d_loss * coef / tokens * logits.shape[1] * counts.max() / counts.sum()
    if got.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * want.abs()
    err = (got.cpu().double() - want).abs()
    assert (err <= tol).all(), (float((err - tol).max()), torch.nonzero(~(err <= tol))[:4].tolist())
    return want


@pytest.mark.parametrize("T,E,K", SIZES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("renormalize", [False, True])
def test_gradient_of_weights_of_small_sigmoids(T, E, K, dtype, renormalize):
    logits = _low_rows(T, E, T + E, dtype)
    dw = torch.randn(T, K, generator=torch.Generator().manual_seed(5))
    router = ep.Router(E, K, scoring=ep.SCORE_SIGMOID, renormalize=renormalize, scale=2.5)
    r = ep.ep_route(logits.cuda(), router)
    got = ep.ep_route_backward(logits.cuda(), router, r, d_weights=dw.cuda())
    want = _compare_gradient(got, logits, r.topk_idx.cpu(), dw, True, renormalize, 2.5)
    if renormalize and K > 1 and dtype == torch.float32:
        assert (want[:16:2].abs().amax(1) > 1e-3).all()         # the rows on trial have a gradient of order one


def _far_picks(T, E, K):
    """A bias that takes K experts in a known order, 85 to 102 below the others; the gaps of the bias outweigh every score."""
    g = torch.Generator().manual_seed(E)
    logits = torch.randn(T, E, generator=g)
    first = E - K - 1 if E > K else 0
    drop = torch.tensor([85.0, 88.0, 91.0, 95.0, 100.0, 102.0])[torch.arange(T) % 6]
    logits[:, first:first + K] = -drop[:, None] + 0.5 * torch.rand(T, K, generator=g)
    bias = torch.zeros(E)
    bias[first:first + K] = 1000.0 - 4.0 * torch.arange(K)
    return logits, bias


@pytest.mark.parametrize("T,E,K", [(30, 8, 3), (30, 24, 4), (30, 60, 6), (24, 256, 8), (24, 300, 5), (16, 1030, 4), (16384, 8, 2), (32768, 16, 4)])
@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("renormalize", [False, True])
def test_gradient_of_picks_that_a_bias_takes_from_far_below(T, E, K, sigmoid, renormalize):
    logits, bias = _far_picks(T, E, K)
    dw = torch.randn(T, K, generator=torch.Generator().manual_seed(6))
    router = ep.Router(E, K, scoring=int(sigmoid), renormalize=renormalize, scale=1.5)
    r = ep.ep_route(logits.cuda(), router, bias=bias.cuda())
    idx = r.topk_idx.cpu()
    assert torch.equal(idx, plain.route(logits, K, sigmoid, bias)[0])
    got = ep.ep_route_backward(logits.cuda(), router, r, d_weights=dw.cuda())
    want = _compare_gradient(got, logits, idx, dw, sigmoid, renormalize, 1.5)
    if renormalize:
        assert (want[:6].abs().amax(1) > 1e-3).all()


@pytest.mark.parametrize("T,E,K", SIZES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_balance_loss_of_small_sigmoids(T, E, K, dtype):
    """A token's probabilities are its scores over their sum, however small the sum is, with and without the picks."""
    logits = _low_rows(T, E, T + E, dtype)
    logits[1::4, E // 2:] -= 95.0                               # scores of a row far apart
    router = ep.Router(E, K, scoring=ep.SCORE_SIGMOID, balance_coef=0.3)
    dev = logits.cuda()
    got = ep.ep_route(dev, router)
    idx = got.topk_idx.cpu()
    _compare_balance(got, logits, idx, True, 0.3)
    table = torch.randint(0, E, (T, K), generator=torch.Generator().manual_seed(3), dtype=torch.int32)
    alone = ep.ep_balance_loss(dev, router, table.cuda())
    _compare_balance(alone, logits, table, True, 0.3)
    d_loss = 50.0
    for r, ids in ((got, idx), (alone, table)):
        grad = ep.ep_route_backward(dev, router, r, d_loss=torch.full((1,), d_loss, device="cuda"))
        _compare_gradient(grad, logits, ids, None, True, True, 1.0, 0.3, d_loss, int(r.tokens), r.expert_counts.cpu().double())


@pytest.mark.parametrize("T,E,K", SIZES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_renormalised_weights_of_small_sigmoids(T, E, K, dtype):
    logits = _low_rows(T, E, T + E, dtype)
    got = ep.ep_route(logits.cuda(), ep.Router(E, K, scoring=ep.SCORE_SIGMOID, scale=2.5))
    idx, w = plain.route(logits, K, True, None, True, 2.5)
    assert torch.equal(got.topk_idx.cpu(), idx)
    assert ((got.topk_weights.cpu().double() - w).abs() <= WEIGHT * w + TINY).all()


@pytest.mark.parametrize("T,E,K", [(30, 8, 3), (30, 24, 4), (30, 60, 6), (24, 256, 8), (24, 300, 5), (16, 1030, 4), (16384, 8, 2), (32768, 16, 4)])
@pytest.mark.parametrize("sigmoid", [False, True])
def test_renormalised_weights_of_picks_that_a_bias_takes_from_far_below(T, E, K, sigmoid):
    logits, bias = _far_picks(T, E, K)
    got = ep.ep_route(logits.cuda(), ep.Router(E, K, scoring=int(sigmoid)), bias=bias.cuda())
    idx, w = plain.route(logits, K, sigmoid, bias)
    assert torch.equal(got.topk_idx.cpu(), idx)
    assert ((got.topk_weights.cpu().double() - w).abs() <= WEIGHT * w + TINY).all()
