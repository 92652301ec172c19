"""The sort, the combine, dropout and the adapters where sizes and surroundings are unusual: buffers past 2^32 bytes, several streams at
once, captured and replayed calls, buffers far larger than what is used."""
import numpy as np
import pytest
import torch

import train_plain as plain
from paper_2609_40093_b200 import ep

pytestmark = pytest.mark.gpu
BF, HALF = torch.bfloat16, 2.0 ** -8
ROWS, WIDE = 300000, 8192                                        # 4.9 GB


def test_rows_past_four_gigabytes():
    big = torch.zeros(ROWS, WIDE, dtype=BF, device="cuda")
    T, K = 3, 2
    slot = torch.tensor([[ROWS - 1, 0], [ROWS - 7, 262145], [-1, ROWS - 2]], dtype=torch.int32, device="cuda")
    x, w = torch.randn(T, WIDE, device="cuda").to(BF), torch.rand(T, K, device="cuda")
    ep.ep_sort(x, slot, big, weights=w)
    for t in range(T):
        for k in range(K):
            if int(slot[t, k]) >= 0:
                assert torch.equal(big[int(slot[t, k])], (x[t].float() * w[t, k]).to(BF))
    y = ep.ep_combine_residual(big, slot, w, torch.empty_like(x))
    sq = torch.where(slot >= 0, w, 0.0).double().square().sum(1, keepdim=True)
    assert float((y.double() - x.double() * sq).norm() / y.double().norm()) < 3 * HALF
    dw = torch.empty(T, K, device="cuda")
    ep.ep_combine_backward(x, slot, w, big, out=big, d_weights=dw)
    want = torch.where(slot >= 0, w.double() * x.double().square().sum(1, keepdim=True), 0.0)
    assert torch.allclose(dw.double(), want, rtol=2 * HALF, atol=0)
    # dropout: the last row, whose vectors are past 2^28, has the bits of its own place
    big.fill_(1.0)
    ep.ep_dropout(big, ep.Dropout(0.5, torch.tensor([21, 4], device="cuda"), 2), y=big)
    first = (ROWS - 1) * (WIDE // 8)
    v = np.arange(first, first + WIDE // 8, dtype=np.uint64)
    c = [v & np.uint64(0xFFFFFFFF), v >> np.uint64(32), np.full(len(v), 4, np.uint64), np.full(len(v), 2, np.uint64)]
    words = plain._rounds(c, 21, 0)
    keep = np.stack([words & 0xFFFF, words >> 16], 2).reshape(-1) >= 32768
    assert np.array_equal(big[-1].float().cpu().numpy(), np.where(keep, 2.0, 0.0))
    # adapters on rows at the end, x and y both past 2^32 bytes
    N, r, A, n = WIDE, 16, 3, 5
    index = torch.tensor([ROWS - 1, 17, ROWS - 3, 270001, ROWS - 2], dtype=torch.int32, device="cuda")
    off = torch.tensor([0, 2, 2, 5], dtype=torch.int32, device="cuda")
    big[index.long()] = torch.randn(n, WIDE, device="cuda").to(BF)
    rows = big[index.long()].clone()
    ad = ep.Adapters((torch.randn(A, r, WIDE, device="cuda") / 90).to(BF), torch.randn(A, N, r, device="cuda").to(BF))
    out = torch.zeros_like(big)
    mid = torch.empty(n, r, dtype=BF, device="cuda")
    ep.ep_adapter_matmul(big, off, ad, out, row_index=index, mid=mid)
    which = torch.tensor([0, 0, 2, 2, 2])
    m = torch.einsum("nh,nrh->nr", rows.double(), ad.down[which].double())
    want = torch.einsum("nr,nor->no", m, ad.up[which].double())
    assert float((out[index.long()].double() - want).norm() / want.norm()) < 2 * HALF
    grads = ep.alloc_adapter_grads(big, ad, entries=n, dx=False)
    ep.ep_adapter_matmul_backward(out, big, off, ad, mid, grads, row_index=index)
    dmid = torch.einsum("no,nor->nr", out[index.long()].double(), ad.up[which].double())
    for a in range(A):
        e = which == a
        down, up = dmid[e].t() @ rows[e].double(), out[index.long()][e].double().t() @ mid[e].double()
        assert float((grads.ddown[a].double() - down).norm()) <= 3 * HALF * float(down.norm())
        assert float((grads.dup[a].double() - up).norm()) <= 2 * HALF * float(up.norm())


def _problem(rows, H, N, r, A, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x, dy, base = (torch.randn(rows, c, generator=g, device="cuda").to(BF) for c in (H, N, N))
    ad = ep.Adapters((torch.randn(A, r, H, generator=g, device="cuda") * H ** -0.5).to(BF), torch.randn(A, N, r, generator=g, device="cuda").to(BF),
                     torch.rand(A, generator=g, device="cuda"))
    ids = torch.randint(-1, A, (rows, 1), generator=g, device="cuda", dtype=torch.int32)
    return x, dy, base, ad, ids


def _all_of_it(x, dy, base, ad, ids, lay, buffers):
    y, mid, grads, ws = buffers
    A = ad.down.shape[0]
    ep.ep_layout(ids, A, 1, out=lay, workspace=ws)
    mid.zero_(), grads.dx.zero_()
    ep.ep_adapter_matmul(x, lay.expert_offsets, ad, y, base=base, row_index=lay.pair_token, mid=mid)
    ep.ep_adapter_matmul_backward(dy, x, lay.expert_offsets, ad, mid, grads, row_index=lay.pair_token)


def _buffers(x, base, ad, ids):
    A, r = ad.down.shape[:2]
    lay = ep.alloc_layout(len(ids), 1, A, 1, fill=-1)
    ws = torch.empty(max(16, ep.ep_layout_workspace_bytes(len(ids), 1, A, 1)), dtype=torch.uint8, device="cuda")
    return lay, (base.clone(), torch.zeros(len(ids), r, dtype=BF, device="cuda"), ep.alloc_adapter_grads(x, ad), ws)


def _results(buffers):
    y, mid, grads, _ = buffers
    return [t.clone() for t in (y, mid, grads.dx, grads.ddown, grads.dup)]


@pytest.mark.parametrize("rows,H,N,r,A", [(300, 512, 768, 16, 20), (4000, 1024, 512, 64, 2)])
def test_two_streams_at_once_and_a_graph(rows, H, N, r, A):
    problems = [_problem(rows, H, N, r, A, s) for s in range(4)]
    want = []
    for p in problems:
        lay, b = _buffers(p[0], p[2], p[3], p[4])
        _all_of_it(*p, lay, b)
        want.append(_results(b))
    torch.cuda.synchronize()
    streams, made = [torch.cuda.Stream() for _ in range(2)], [_buffers(p[0], p[2], p[3], p[4]) for p in problems]
    torch.cuda.synchronize()
    for _ in range(5):
        for i, (p, (lay, b)) in enumerate(zip(problems, made)):
            with torch.cuda.stream(streams[i % 2]):
                _all_of_it(*p, lay, b)
    torch.cuda.synchronize()
    for (lay, b), w in zip(made, want):
        assert all(torch.equal(g, t) for g, t in zip(_results(b), w))
    # captured on one problem, replayed on the others: the tensors' contents change, ids among them
    x, dy, base, ad, ids = (problems[0][i].clone() if i != 3 else ep.Adapters(*(t.clone() for t in (problems[0][3].down, problems[0][3].up, problems[0][3].scale)))
                            for i in range(5))
    lay, b = _buffers(x, base, ad, ids)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _all_of_it(x, dy, base, ad, ids, lay, b)
    for p, w in zip(problems, want):
        x.copy_(p[0]), dy.copy_(p[1]), base.copy_(p[2]), ids.copy_(p[4])
        ad.down.copy_(p[3].down), ad.up.copy_(p[3].up), ad.scale.copy_(p[3].scale)
        b[0].copy_(base)
        graph.replay()
        assert all(torch.equal(g, t) for g, t in zip(_results(b), w))


def test_beside_the_experts_products_on_another_stream():
    """Both kinds of kernel take tensor memory; clusters of either wait for each other's CTAs only."""
    x, dy, base, ad, ids = _problem(64, 2048, 2048, 16, 16, 9)
    lay, b = _buffers(x, base, ad, ids)
    g = torch.Generator(device="cuda").manual_seed(1)
    w = (torch.randn(8, 1024, 2048, generator=g, device="cuda") / 45).to(BF)
    rows = torch.randn(512, 2048, generator=g, device="cuda").to(BF)
    off = (torch.arange(9, device="cuda") * 64).int()
    _all_of_it(x, dy, base, ad, ids, lay, b)
    want, out = _results(b), ep.ep_expert_matmul(rows, off, w)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    other, got = torch.cuda.Stream(), torch.empty_like(out)
    torch.cuda.synchronize()
    for _ in range(50):
        with torch.cuda.stream(other):
            ep.ep_expert_matmul(rows, off, w, y=got, status=status)
        _all_of_it(x, dy, base, ad, ids, lay, b)
    torch.cuda.synchronize()
    assert torch.equal(got, out) and int(status) == 0 and all(torch.equal(a, c) for a, c in zip(_results(b), want))


def test_few_entries_in_large_buffers():
    """The launches follow the buffers' size; what is not used is neither read nor written."""
    rows, H, N, r, A = 20000, 256, 264, 24, 6
    x = torch.full((rows, H), float("nan"), dtype=BF, device="cuda")
    y = torch.full((rows, N), 3.0, dtype=BF, device="cuda")
    x[:70] = torch.randn(70, H, device="cuda").to(BF)
    ad = ep.Adapters((torch.randn(A, r, H, device="cuda") / 16).to(BF), torch.randn(A, N, r, device="cuda").to(BF))
    off = torch.tensor([0, 0, 69, 69, 70, 70, 70], dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    mid = torch.full((rows, r), 5.0, dtype=BF, device="cuda")
    ep.ep_adapter_matmul(x, off, ad, y, base=y, mid=mid, status=status)
    for a, e in ((1, slice(0, 69)), (3, slice(69, 70))):
        m = x[e].double() @ ad.down[a].double().t()
        want = 3.0 + m @ ad.up[a].double().t()
        assert float((y[e].double() - want).norm() / want.norm()) < 2 * HALF
    assert (y[70:] == 3).all() and (mid[70:] == 5).all()
    grads = ep.alloc_adapter_grads(x, ad)
    grads.dx.fill_(2.0)
    dy = torch.full((rows, N), float("nan"), dtype=BF, device="cuda")
    dy[:70] = torch.randn(70, N, device="cuda").to(BF)
    mid[70:] = float("nan")
    ep.ep_adapter_matmul_backward(dy, x, off, ad, mid, grads, base=grads.dx, status=status)
    assert (grads.dx[70:] == 2).all() and all(torch.isfinite(t).all() for t in (grads.dx, grads.ddown, grads.dup))
    for a, e in ((1, slice(0, 69)), (3, slice(69, 70))):
        up = dy[e].double().t() @ mid[e].double()
        down = (dy[e].double() @ ad.up[a].double()).t() @ x[e].double()
        assert float((grads.dup[a].double() - up).norm() / up.norm()) < 2 * HALF
        assert float((grads.ddown[a].double() - down).norm() / down.norm()) < 3 * HALF
    for a in (0, 2, 4, 5):
        assert (grads.ddown[a] == 0).all() and (grads.dup[a] == 0).all()
    assert int(status) == 0
