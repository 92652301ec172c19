"""Router, balance loss and their gradient on the GPU against the 64-bit statements of `moe_plain`.

Tolerances, all fp32 arithmetic with u = 2^-24. A score is an exponential (2 ulp), a sum of E positive terms (warp tree
and at most E/32 terms a lane: relative error below (E/32 + 5) u) and a division: relative error below (E/32 + 16) u; the
argument l - max of the exponential is rounded (u * |l - max|, at most 200 here where the score is not negligible). Weights,
probabilities: WEIGHT = 2^-15 relative covers E up to 4096, plus 1e-7 absolute for terms whose relative error the argument's
rounding dominates. Gradients are sums of products of such terms, no larger than the largest |d_weights| * scale / (sum of
the picked scores): 2^-14 of the row's largest absolute term. bf16 logits: the gradient is rounded once more, 2^-8 relative."""
import math

import pytest
import torch

import moe_plain as plain
from paper_2609_40093_b200 import ep

pytestmark = pytest.mark.gpu

WEIGHT, TINY = 2.0 ** -15, 1e-7


def _logits(T, E, dtype, seed, spread=1.5):
    g = torch.Generator().manual_seed(seed)
    return (spread * torch.randn(T, E, generator=g) + 0.7 * torch.randn(E, generator=g)).to(dtype)


def _compare_route(logits, router, bias=None, order_by=None):
    got = ep.ep_route(logits.cuda(), router, bias=None if bias is None else bias.cuda())
    sig = router.scoring == ep.SCORE_SIGMOID
    idx, w = plain.route(logits, router.top_k, sig, bias, router.renormalize, router.scale, order_by)
    assert torch.equal(got.topk_idx.cpu(), idx)
    assert ((got.topk_weights.cpu().double() - w).abs() <= WEIGHT * w.abs() + TINY).all()
    return got, idx


SIZES = [(1, 1, 1), (1, 8, 2), (300, 8, 8), (5, 7, 9), (257, 13, 4), (40, 16, 16), (31, 16, 3), (40, 17, 5), (3, 4, 4), (64, 8, 2), (5, 31, 3), (4, 32, 32), (9, 33, 5), (7, 60, 6), (17, 64, 8), (33, 127, 7),
         (20, 128, 8), (257, 256, 8), (13, 257, 4), (6, 510, 10), (8, 512, 10), (3, 1000, 8), (2, 1025, 3), (3, 2044, 9), (2, 4096, 32)]


@pytest.mark.parametrize("T,E,K", SIZES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sigmoid", [False, True])
def test_picks_and_weights(T, E, K, dtype, sigmoid):
    logits = _logits(T, E, dtype, T * E + K)
    for renormalize, scale in ((True, 1.0), (False, 2.5)):
        _compare_route(logits, ep.Router(E, K, scoring=int(sigmoid), renormalize=renormalize, scale=scale))


@pytest.mark.parametrize("T,E,K", [(2048, 1, 1), (6200, 3, 3), (10241, 5, 7), (16384, 8, 2), (16500, 8, 8), (23000, 11, 3), (26700, 13, 1), (32769, 16, 16)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("renormalize", [False, True])
def test_many_tokens_on_few_experts(T, E, K, dtype, sigmoid, renormalize):
    """Picks, weights, loss and gradient where a thread takes a token: masked tokens and experts, NaN, ties (coarse logits)."""
    logits = _logits(T, E, torch.float32, T + E)
    logits[::3] = (logits[::3] * 2).round() / 2
    logits[torch.rand(T, generator=torch.Generator().manual_seed(E)) < 0.05] = -math.inf
    logits[5, 0] = math.nan
    logits[7, E - 1] = math.inf
    logits[9] = torch.finfo(torch.float32).min if dtype == torch.float32 else -1e38
    logits = logits.to(dtype)
    router = ep.Router(E, K, scoring=int(sigmoid), renormalize=renormalize, scale=1.5, balance_coef=0.4)
    got, idx = _compare_route(logits, router)
    assert int(got.status) == ep.STATUS_BAD_LOGIT
    _compare_balance(got, logits, idx, sigmoid, 0.4)
    plain_call = ep.ep_route(logits.cuda(), router, out=ep.alloc_routing(T, E, K))
    assert torch.equal(plain_call.topk_idx, got.topk_idx) and torch.equal(plain_call.topk_weights, got.topk_weights)
    table = idx.clone()
    table[11] = -1
    alone = ep.ep_balance_loss(logits.cuda(), router, table.cuda())
    _compare_balance(alone, logits, table, sigmoid, 0.4)
    dw, dl = torch.randn(T, K, generator=torch.Generator().manual_seed(1)), 700.0
    grad = ep.ep_route_backward(logits.cuda(), router, got, d_weights=dw.cuda(), d_loss=torch.full((1,), dl, device="cuda"))
    want = plain.route_gradient(logits, idx, dw, sigmoid, renormalize, 1.5, 0.4, dl)
    s = plain.scores(logits, sigmoid)[0]
    picked = torch.where(idx >= 0, torch.gather(s, 1, idx.clamp(min=0).long()), 0.0)
    unit = 1.5 / (picked.sum(1, keepdim=True).clamp(min=1e-300) if renormalize else torch.ones(T, 1, dtype=torch.float64))
    largest = (dw.double().abs() * unit * picked).amax(1, keepdim=True)
    counts = got.expert_counts.cpu().double()
    share = dl * 0.4 / int(got.tokens) * E * counts.max() / counts.sum()
    tol = 2.0 ** -14 * (largest + share) + 1e-30 + (2.0 ** -8 * want.abs() if dtype == torch.bfloat16 else 0.0)
    assert ((grad.cpu().double() - want).abs() <= tol).all()
    bias = (torch.randint(-8, 9, (E,), generator=torch.Generator().manual_seed(2)).float() * 4)    # outweighs every score: orders alone
    biased = ep.ep_route(logits.cuda(), router, bias=bias.cuda(), out=ep.alloc_routing(T, E, K, balance=True))
    ids = biased.topk_idx.cpu()
    order = torch.where(plain.masked(logits), -math.inf, (s + bias.double()))
    ranked = torch.gather(order, 1, ids.clamp(min=0).long())
    assert (ranked[:, :-1] >= ranked[:, 1:] - 1e-6).masked_fill(ids[:, 1:] < 0, True).all()
    assert torch.equal((ids >= 0).sum(1), (order > -math.inf).sum(1).clamp(max=K))
    _compare_balance(biased, logits, ids, sigmoid, 0.4)


def test_equal_logits_go_to_the_lowest_expert():
    E, K = 96, 6
    logits = torch.zeros(40, E)
    logits[1] = 7.0
    logits[2, ::2] = -0.0                                       # -0 equals +0
    logits[3:] = torch.randint(-2, 3, (37, E), generator=torch.Generator().manual_seed(1)).float()
    for dtype in (torch.float32, torch.bfloat16):
        for sigmoid in (0, 1):
            got, _ = _compare_route(logits.to(dtype), ep.Router(E, K, scoring=sigmoid))
            assert got.topk_idx[0].tolist() == got.topk_idx[1].tolist() == got.topk_idx[2].tolist() == list(range(K))


@pytest.mark.parametrize("E", [8, 60, 256, 1030])
@pytest.mark.parametrize("sigmoid", [False, True])
def test_masked_rows_experts_and_extreme_logits(E, sigmoid):
    K = 4
    logits = _logits(12, E, torch.float32, E)
    logits[0] = -math.inf                                       # nothing left
    logits[1, 3:] = -math.inf                                   # fewer experts than picks
    logits[2] = torch.finfo(torch.float32).min                  # the type's lowest value is a logit, not a mask
    logits[3, : E // 2] = torch.finfo(torch.float32).min
    logits[4] = 3.0e38
    logits[5, 1] = 3.0e38
    logits[6] = -100.0                                          # sigmoids that underflow to almost nothing
    logits[7, ::2] = -math.inf
    for renormalize in (True, False):
        got, idx = _compare_route(logits, ep.Router(E, K, scoring=int(sigmoid), renormalize=renormalize))
        assert int(got.status) == 0
        assert got.topk_idx[0].tolist() == [-1] * K and got.topk_weights[0].abs().max() == 0
        assert got.topk_idx[1].tolist()[3:] == [-1] and got.topk_weights[1, 3] == 0
        assert torch.isfinite(got.topk_weights).all()


@pytest.mark.parametrize("sigmoid", [False, True])
def test_nan_and_inf_logits_are_not_picked_and_are_reported(sigmoid):
    E, K = 40, 5
    for bad in (math.nan, math.inf):
        logits = _logits(9, E, torch.float32, 2)
        logits[4, 7] = bad
        got, idx = _compare_route(logits, ep.Router(E, K, scoring=int(sigmoid), balance_coef=0.1))
        assert int(got.status) == ep.STATUS_BAD_LOGIT
        assert torch.isfinite(got.mean_probs).all() and torch.isfinite(got.loss).all()
        logits[4] = bad
        got = ep.ep_route(logits.cuda(), ep.Router(E, K, scoring=int(sigmoid)))
        assert got.topk_idx[4].tolist() == [-1] * K


@pytest.mark.parametrize("T,E,K", [(1, 8, 2), (64, 60, 6), (130, 256, 8), (5, 1100, 4)])
@pytest.mark.parametrize("sigmoid", [False, True])
def test_selection_bias_orders_but_does_not_weigh(T, E, K, sigmoid):
    """Scores on a coarse grid of logits and a bias of whole numbers of 2^-6 far outweighing fp32's rounding: the order does
    not hang on the last bits, and equal sums (which occur) still go to the lowest expert in both."""
    g = torch.Generator().manual_seed(E)
    logits = torch.randint(-3, 4, (T, E), generator=g).float()
    bias = torch.randint(-8, 9, (E,), generator=g).float() / 64 * (1.0 if sigmoid else 64.0)
    logits[0, 0] = -math.inf
    s = plain.scores(logits, sigmoid)[0]
    order = torch.round((s + bias.double()) * 2 ** 18)         # equal iff the fp32 sums are: distinct ones differ by far more
    for row in order:                                           # within a token: picks of different tokens are not compared
        distinct = torch.unique(row)
        # sums below 16 are rounded by at most 2^-21 in fp32, scores by less: two steps of 2^-18 keep distinct ones apart
        assert len(distinct) == 1 or distinct.diff().min() >= 2
    router = ep.Router(E, K, scoring=int(sigmoid), scale=2.0)
    if sigmoid:
        _compare_route(logits, router, bias)
    else:                                                       # softmax scores of equal logits are equal bits in a row
        got = ep.ep_route(logits.cuda(), router, bias=bias.cuda())
        idx, w = plain.route(logits, K, False, bias, True, 2.0)
        assert torch.equal(got.topk_idx.cpu(), idx)
        assert ((got.topk_weights.cpu().double() - w).abs() <= WEIGHT * w + TINY).all()
    shut = bias.clone()
    shut[1 % E] = -math.inf                                     # a bias of -inf masks the expert as well
    got = ep.ep_route(logits.cuda(), router, bias=shut.cuda())
    assert not (got.topk_idx == 1 % E).any() and int(got.status) == 0


BALANCE = [(1, 8, 2), (64, 8, 2), (700, 5, 2), (3000, 16, 4), (333, 11, 3), (50, 17, 3), (300, 60, 6), (1000, 128, 8), (97, 257, 4), (2500, 256, 8), (40, 1030, 8), (9, 4096, 32)]


def _compare_balance(got, logits, idx, sigmoid, coef):
    counts, n, mean, loss = plain.balance(logits, idx, sigmoid, coef)
    assert torch.equal(got.expert_counts.cpu(), counts) and int(got.tokens) == n
    assert ((got.mean_probs.cpu().double() - mean).abs() <= WEIGHT * mean + 1e-9).all()
    assert abs(float(got.loss) - float(loss)) <= 2 * WEIGHT * abs(float(loss))


@pytest.mark.parametrize("T,E,K", BALANCE)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sigmoid", [False, True])
def test_balance_loss_with_and_without_the_picks(T, E, K, dtype, sigmoid):
    logits = _logits(T, E, dtype, 7 * T + E)
    logits[torch.rand(T, generator=torch.Generator().manual_seed(T)) < 0.1] = -math.inf
    router = ep.Router(E, K, scoring=int(sigmoid), balance_coef=0.02)
    dev = logits.cuda()
    got = ep.ep_route(dev, router)
    idx = got.topk_idx.cpu()
    _compare_balance(got, logits, idx, sigmoid, 0.02)
    again = ep.ep_route(dev, router, out=ep.alloc_routing(T, E, K, balance=True))
    for f in ("topk_idx", "topk_weights", "expert_counts", "mean_probs", "loss"):
        assert torch.equal(getattr(got, f), getattr(again, f)), f                       # the same bits every time
    # a table from elsewhere: masked and out-of-range entries, a row without a pick
    other = torch.randint(0, E, (T, K), generator=torch.Generator().manual_seed(3), dtype=torch.int32)
    other[T // 2] = -1
    if K > 1:
        other[0, 1] = -1
    alone = ep.ep_balance_loss(dev, router, other.cuda())
    _compare_balance(alone, logits, other, sigmoid, 0.02)
    assert int(alone.status) == 0
    other[0, 0] = E + 3
    alone = ep.ep_balance_loss(dev, router, other.cuda())
    _compare_balance(alone, logits, other, sigmoid, 0.02)
    assert int(alone.status) == ep.STATUS_BAD_INDEX


def test_balance_of_nothing_is_zero():
    router = ep.Router(16, 2, balance_coef=1.0)
    for T in (0, 3):
        logits = torch.full((T, 16), -math.inf, device="cuda")
        got = ep.ep_route(logits, router)
        assert got.expert_counts.abs().sum() == 0 and got.mean_probs.abs().sum() == 0 and float(got.loss) == 0 and int(got.tokens) == 0
        d = ep.ep_route_backward(logits, router, got, d_weights=torch.ones(T, 2, device="cuda"), d_loss=torch.ones(1, device="cuda"))
        assert d.shape == (T, 16) and d.abs().sum() == 0


@pytest.mark.parametrize("T,E,K", [(1, 8, 2), (64, 8, 8), (300, 5, 2), (77, 16, 5), (30, 11, 11), (50, 60, 6), (200, 128, 8), (33, 257, 4), (300, 256, 8), (12, 1030, 8), (4, 4096, 32)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("renormalize", [False, True])
def test_gradient(T, E, K, dtype, sigmoid, renormalize):
    logits = _logits(T, E, dtype, T + E)
    logits[torch.rand(T, generator=torch.Generator().manual_seed(E)) < 0.1] = -math.inf
    logits[0, E // 2] = -math.inf
    if T > 2:
        logits[2, 0] = math.nan
    g = torch.Generator().manual_seed(11)
    dw = torch.randn(T, K, generator=g)
    router = ep.Router(E, K, scoring=int(sigmoid), renormalize=renormalize, scale=2.5, balance_coef=0.7)
    dev = logits.cuda()
    r = ep.ep_route(dev, router)
    idx = r.topk_idx.cpu()
    d_loss = torch.tensor([1.3])
    s = plain.scores(logits, sigmoid)[0]
    picked = torch.where(idx >= 0, torch.gather(s, 1, idx.clamp(min=0).long()), 0.0)
    unit = 2.5 / (picked.sum(1, keepdim=True).clamp(min=1e-300) if renormalize else torch.ones(T, 1, dtype=torch.float64))
    largest = (dw.double().abs() * unit * picked).amax(1, keepdim=True)
    for weights, loss in ((True, True), (True, False), (False, True)):
        got = ep.ep_route_backward(dev, router, r, d_weights=dw.cuda() if weights else None, d_loss=d_loss.cuda() if loss else None)
        want = plain.route_gradient(logits, idx, dw if weights else None, sigmoid, renormalize, 2.5, 0.7 if loss else 0.0, 1.3)
        assert got.dtype == dtype
        err = (got.cpu().double() - want).abs()
        counts = r.expert_counts.cpu().double()
        share = 1.3 * 0.7 / max(1, int(r.tokens)) * E * counts.max() / max(1, int(counts.sum()))    # largest gradient of a probability
        tol = 2.0 ** -14 * ((largest if weights else 0.0) + (share if loss else 0.0)) + 1e-30
        if dtype == torch.bfloat16:
            tol = tol + 2.0 ** -8 * want.abs()
        assert (err <= tol).all(), float((err - tol).max())
        assert (got.cpu()[plain.masked(logits)] == 0).all()


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("renormalize", [False, True])
def test_gradient_against_differences_of_the_kernel(sigmoid, renormalize):
    """<gradient, d> against (L(l + h d) - L(l - h d)) / 2h of the kernel's own outputs, summed in 64 bits. With h = 2^-6 the
    difference's truncation error is h^2 / 6 times a third derivative (below 3e-4 of the sum of |terms|), fp32 rounding of
    the outputs gives 2^-22 / h = 2^-16 of it."""
    T, E, K = 64, 24, 4
    g = torch.Generator().manual_seed(8)
    logits = 2.0 * torch.randn(T, E, generator=g)
    logits = (logits * 64).round() / 64
    top = logits.sort(1, descending=True).values
    keep = (top[:, K - 1] - top[:, K]) > 0.25                   # picks that do not change within h
    logits, d = logits[keep].cuda().contiguous(), (torch.randint(0, 2, logits[keep].shape, generator=g) * 2 - 1).float().cuda()
    T = logits.shape[0]
    assert T > 16
    dw = torch.randn(T, K, generator=g).cuda()
    router = ep.Router(E, K, scoring=int(sigmoid), renormalize=renormalize, balance_coef=5.0)
    r = ep.ep_route(logits, router)
    base = r.topk_idx.clone()
    grad = ep.ep_route_backward(logits, router, r, d_weights=dw, d_loss=torch.ones(1, device="cuda"))

    def objective(l):
        q = ep.ep_route(l, router)
        slot = (q.topk_idx[:, :, None] == base[:, None, :]).double()           # a pick may change its place within the row
        assert slot.sum() == T * K
        return float((torch.einsum("tk,tkj->tj", q.topk_weights.double(), slot) * dw.double()).sum() + q.loss.double())

    h = 2.0 ** -6
    want = (objective(logits + h * d) - objective(logits - h * d)) / (2 * h)
    got = float((grad.double() * d.double()).sum())
    size = float((grad.double().abs()).sum())
    assert abs(got - want) <= 1e-3 * size, (got, want, size)


def test_unaligned_rows_other_streams_and_graphs():
    T, E, K = 77, 64, 6
    router = ep.Router(E, K, balance_coef=0.1)
    logits = _logits(T, E, torch.float32, 1)
    want = ep.ep_route(logits.cuda(), router)
    dw, dl = torch.randn(T, K, device="cuda"), torch.ones(1, device="cuda")
    dwant = ep.ep_route_backward(logits.cuda(), router, want, d_weights=dw, d_loss=dl)
    shifted = torch.empty(T * E + 1, device="cuda")[1:].view(T, E)                      # 4-byte aligned only
    shifted.copy_(logits)
    dshift = torch.empty(T * E + 1, device="cuda")[1:].view(T, E)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = ep.ep_route(shifted, router)
        ep.ep_route_backward(shifted, router, got, d_weights=dw, d_loss=dl, dlogits=dshift)
    torch.cuda.current_stream().wait_stream(side)
    for f in ("topk_idx", "topk_weights", "expert_counts", "tokens", "mean_probs", "loss"):
        assert torch.equal(getattr(got, f), getattr(want, f)), f
    assert torch.equal(dshift, dwant)
    static, out, grad = logits.cuda(), ep.alloc_routing(T, E, K, balance=True), torch.empty(T, E, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ep.ep_route(static, router, out=out)
        ep.ep_route_backward(static, router, out, d_weights=dw, d_loss=dl, dlogits=grad)
    for seed in (5, 6):
        static.copy_(_logits(T, E, torch.float32, seed))
        graph.replay()
        fresh = ep.ep_route(static, router)
        assert torch.equal(out.topk_idx, fresh.topk_idx) and torch.equal(out.loss, fresh.loss)
        assert torch.equal(grad, ep.ep_route_backward(static, router, fresh, d_weights=dw, d_loss=dl))


@pytest.mark.parametrize("E", [8, 13, 24, 256])
def test_tokens_that_a_bias_leaves_without_an_expert_are_not_counted(E):
    T, K = 20, 3
    logits = _logits(T, E, torch.float32, 2)
    logits[:7, 4:] = -math.inf                                  # seven tokens know only experts 0 to 3 ...
    bias = torch.zeros(E)
    bias[:4] = -math.inf                                        # ... which are shut
    router = ep.Router(E, K, scoring=ep.SCORE_SIGMOID, balance_coef=0.3)
    got = ep.ep_route(logits.cuda(), router, bias=bias.cuda(), out=ep.alloc_routing(T, E, K, balance=True))
    idx = got.topk_idx.cpu()
    assert (idx[:7] == -1).all() and (idx[7:] >= 4).all()
    _compare_balance(got, logits, idx, True, 0.3)
    d = ep.ep_route_backward(logits.cuda(), router, got, d_weights=torch.ones(T, K, device="cuda"), d_loss=torch.ones(1, device="cuda"))
    assert d[:7].abs().sum() == 0 and torch.isfinite(d).all()


def test_outputs_stay_inside_their_buffers():
    T, E, K = 131, 60, 7
    router = ep.Router(E, K, balance_coef=0.1)
    logits = _logits(T, E, torch.bfloat16, 4).cuda()
    nws = ep.ep_route_workspace_bytes(T, K, E)
    whole = {}

    def carve(name, dtype, *shape, fill=77):
        n = math.prod(shape)
        whole[name] = torch.full((n + 32,), 77, dtype=dtype, device="cuda")
        whole[name][16:16 + n] = fill
        return whole[name][16:16 + n].view(*shape)

    out = ep.Routing(carve("idx", torch.int32, T, K), carve("w", torch.float32, T, K), torch.zeros(1, dtype=torch.int32, device="cuda"),
                     carve("counts", torch.int32, E), carve("tokens", torch.int32, 1), carve("mean", torch.float32, E),
                     carve("loss", torch.float32, 1), carve("ws", torch.uint8, nws, fill=0))
    ep.ep_route(logits, router, out=out)
    grad = carve("grad", torch.bfloat16, T, E)
    ep.ep_route_backward(logits, router, out, d_weights=torch.ones(T, K, device="cuda"), d_loss=torch.ones(1, device="cuda"), dlogits=grad)
    for name, t in whole.items():
        assert (t[:16] == 77).all() and (t[-16:] == 77).all(), name
    assert (out.workspace == 0).all()                           # left for the next call as it was found


def test_a_large_table_agrees_with_its_parts():
    """65536 x 256 against the same rows routed in four parts: the same picks, weights and gradients, and sums that add up."""
    T, E, K = 65536, 256, 8
    router = ep.Router(E, K, scoring=ep.SCORE_SIGMOID, balance_coef=0.0)
    g = torch.Generator(device="cuda").manual_seed(0)
    logits = torch.randn(T, E, device="cuda", generator=g)
    whole = ep.ep_route(logits, router, out=ep.alloc_routing(T, E, K, balance=True))
    parts = [ep.ep_route(logits[i:i + 16384], router, out=ep.alloc_routing(16384, E, K, balance=True)) for i in range(0, T, 16384)]
    assert torch.equal(whole.topk_idx, torch.cat([p.topk_idx for p in parts]))
    assert torch.equal(whole.topk_weights, torch.cat([p.topk_weights for p in parts]))
    assert torch.equal(whole.expert_counts, sum(p.expert_counts for p in parts)) and int(whole.expert_counts.sum()) == T * K
    mean = sum(p.mean_probs.double() for p in parts) / 4
    assert ((whole.mean_probs.double() - mean).abs() <= WEIGHT * mean).all()


def test_tensors_of_a_routing_may_be_exchanged_between_calls():
    """What a Routing remembers of its tensors is forgotten when one is replaced or moves."""
    T, E, K = 40, 16, 2
    router, logits = ep.Router(E, K, balance_coef=0.1), _logits(40, 16, torch.float32, 3).cuda()
    out = ep.ep_route(logits, router)
    idx = out.topk_idx.clone()
    fresh = torch.full_like(idx, -7)
    out.topk_idx = fresh
    ep.ep_route(logits, router, out=out)
    assert torch.equal(fresh, idx)
    out.topk_idx = torch.zeros(T, K, dtype=torch.int64, device="cuda")
    with pytest.raises(TypeError, match="topk_idx"):
        ep.ep_route(logits, router, out=out)
    out.topk_idx = fresh
    out.mean_probs.resize_(4 * E)                               # other memory behind the same tensor, of another shape
    with pytest.raises(ValueError, match="mean_probs"):
        ep.ep_route(logits, router, out=out)
