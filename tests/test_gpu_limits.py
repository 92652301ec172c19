"""The ends of the documented ranges: token and row counts just below 2^31, where a rounded-up quotient in 32 bits would overflow."""
import pytest
import torch

from paper_2609_40093_b200 import ep

pytestmark = pytest.mark.gpu

MOST = 2 ** 31 - 1
CHUNK = 1 << 28


def _room(gigabytes):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gigabytes * 10 ** 9:
        pytest.skip(f"needs {gigabytes} GB of device memory")


def _pieces(t):
    return (t[i:i + CHUNK] for i in range(0, t.shape[0], CHUNK))


def test_most_tokens_on_one_expert():
    """One pick per token: T * K is the largest that is allowed. A thread per token; picks, loss and gradient."""
    _room(45)
    logits = torch.empty(MOST, 1, dtype=torch.bfloat16, device="cuda")
    values = torch.tensor([-3.0, -1.5, 0.0, 0.5, 2.0], dtype=torch.bfloat16, device="cuda")
    period = values.repeat(CHUNK // 5 + 1)
    for i, piece in enumerate(_pieces(logits)):
        start = i * CHUNK % 5
        piece[:, 0] = period[start:start + piece.shape[0]]
    router = ep.Router(1, 1, scoring=ep.SCORE_SIGMOID, renormalize=False, balance_coef=0.25)
    r = ep.ep_route(logits, router, out=ep.alloc_routing(MOST, 1, 1))

    def holds(t, of):
        for x, piece in zip(_pieces(logits), _pieces(t)):
            for v, w in zip(values, of):
                got = piece[x == v].double()
                if not ((got - w).abs() <= 2.0 ** -8 * w.abs()).all():
                    return False
        return True

    want = torch.sigmoid(values.double())
    assert all((p == 0).all() for p in _pieces(r.topk_idx)) and holds(r.topk_weights, want)
    r = ep.ep_route(logits, router)
    assert int(r.expert_counts) == MOST and int(r.tokens) == MOST
    assert abs(float(r.mean_probs) - 1.0) < 2.0 ** -15 and abs(float(r.loss) - 0.25) < 2.0 ** -15
    again = ep.ep_balance_loss(logits, router, r.topk_idx)
    assert int(again.expert_counts) == MOST and abs(float(again.loss) - 0.25) < 2.0 ** -15
    r.topk_weights.fill_(1.0)                                   # the gradient's d_weights
    grad = ep.ep_route_backward(logits, router, r, d_weights=r.topk_weights)
    assert holds(grad, want * (1 - want))


def test_most_tokens_on_some_experts():
    """A warp per token."""
    _room(100)
    logits = torch.zeros(MOST, 17, dtype=torch.bfloat16, device="cuda")
    r = ep.ep_route(logits, ep.Router(17, 1, renormalize=False))
    assert all((p == 0).all() for p in _pieces(r.topk_idx))
    assert all(((p - 1 / 17).abs() < 1e-7).all() for p in _pieces(r.topk_weights))


@pytest.mark.parametrize("cut", [[], [MOST - 300], [5, 2 ** 30, MOST - 1]], ids=str)
def test_most_rows_of_the_experts_products(cut):
    """2^31 - 1 rows of eight features, nearly all of them zero: every row is written, those next to the bounds are right."""
    _room(75)
    bounds = [0] + cut + [MOST]
    E = len(bounds) - 1
    x = torch.zeros(MOST, 8, dtype=torch.bfloat16, device="cuda")
    y = torch.full((MOST, 8), 31.0, dtype=torch.bfloat16, device="cuda")
    w = torch.stack([torch.eye(8) * (e + 2) for e in range(E)]).bfloat16().cuda()
    marked = sorted({0, 1, 12345, 2 ** 30 + 7, MOST - 1, MOST - 2} | {b + d for b in cut for d in (-1, 0)})
    for p in marked:
        x[p] = torch.arange(8) + 1
    ep.ep_expert_matmul(x, torch.tensor(bounds, dtype=torch.int32, device="cuda"), w, y=y)
    for p in marked:
        e = max(i for i in range(E) if bounds[i] <= p)
        assert y[p].tolist() == [(e + 2.0) * (i + 1) for i in range(8)], p
    assert sum(int(torch.count_nonzero(piece)) for piece in _pieces(y)) == 8 * len(marked)
