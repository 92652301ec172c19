"""ep_sort, ep_sort_backward, ep_combine_residual, ep_combine_backward and ep_dropout against their plain statements in 64 bits.

Tolerances: a result in bf16 is one rounding of an fp32 value, half a step of it (2^-8); an fp32 sum of n terms is off by at most n 2^-24 of
the sum of their magnitudes (n + 4 with the products' and the scale's own roundings); 2^-133 covers the smallest bf16 numbers."""
import pytest
import torch

import train_plain as plain
from gpu_util import guarded, guards_intact
from paper_2609_40093_b200 import ep

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def _within(got, want, mag, terms, half=2.0 ** -8):
    got, err = got.double().cpu(), (terms + 4) * 2.0 ** -24 * mag
    assert torch.isfinite(got).all()
    bad = (got - want).abs() > half * (want.abs() + err) + err + 2.0 ** -133
    assert not bad.any(), (int(bad.sum()), float((got - want).abs().max()))


def _slots(T, K, rows, g, masked, shared):
    """Distinct rows (as pair_slot); shared: picks of a token may name one row (as recv_slot)."""
    slot = torch.randperm(rows, generator=g)[:T * K].view(T, K)
    if shared:
        pick = torch.randint(0, K, (T, K), generator=g)
        slot = torch.where(torch.rand(T, K, generator=g) < 0.5, torch.gather(slot, 1, pick), slot)
    slot = torch.where(torch.rand(T, K, generator=g) < masked, -1, slot)
    if T > 2:
        slot[T // 2] = -1                                        # a token whose mask leaves nothing
    return slot


def _data(T, K, H, seed, masked=0.2, shared=False, spare=3):
    g = torch.Generator().manual_seed(seed)
    rows = T * K + spare
    slot = _slots(T, K, rows, g, masked, shared)
    w = torch.softmax(torch.randn(T, K, generator=g), 1)
    w = torch.where(slot < 0, float("nan"), w)                   # what a masked pick's weight holds must not matter
    table, x, add = (torch.randn(n, H, generator=g).to(BF) for n in (rows, T, T))
    named = torch.zeros(rows, dtype=torch.bool)
    named[slot[slot >= 0]] = True
    table[~named] = float("nan")                                 # nor what unnamed rows hold
    return slot, w, table, x, add, named


SHAPES = [(1, 1, 8), (3, 2, 264), (64, 2, 512), (37, 6, 520), (130, 8, 2048), (33, 8, 2056), (5, 9, 72), (19, 16, 1032), (7, 32, 136), (9, 17, 2064), (2, 11, 6304), (149, 3, 1096), (700, 1, 1032)]


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("T,K,H", SHAPES)
def test_sort_and_its_gradients(T, K, H, shared):
    slot, w, table, x, add, named = _data(T, K, H, T + K + H, shared=shared)
    rows, s, xd, td = table.shape[0], slot.int().cuda(), x.cuda(), table.cuda()
    wd, w64 = w.cuda(), torch.where(slot >= 0, w.double(), 0.0)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    whole, out = guarded(rows, H)
    before = out.clone()
    ep.ep_sort(xd, s, out, weights=wd, status=status)
    want, _ = plain.spread(x.double(), slot, w64, rows)
    mag, _ = plain.spread(x.double().abs(), slot, w64, rows)
    _within(out[named.cuda()], want[named], mag[named], K)
    assert torch.equal(out[~named.cuda()].view(torch.int16), before[~named.cuda()].view(torch.int16)) and guards_intact(whole)
    plain_rows = torch.full((rows, H), 7.0, dtype=BF, device="cuda")      # without weights: the row itself
    ep.ep_sort(xd, s, plain_rows, status=status)
    assert torch.equal(plain_rows, ep.ep_dispatch(xd, s, torch.full_like(plain_rows, 7.0), 1, 1))

    finite = torch.where(named[:, None], table.double(), 0.0)
    for weights, w_64 in ((wd, w64), (None, None)):
        for extra in (None, add.cuda()):
            dx = torch.empty(T, H, dtype=BF, device="cuda")
            dw = torch.full((T, K), 9.0, device="cuda") if weights is not None else None
            ep.ep_sort_backward(td, s, dx, weights=weights, x=xd if weights is not None else None, d_weights=dw, add=extra, status=status)
            want, mag = plain.gather(finite, slot, w_64)
            if extra is not None:
                want, mag = want + add.double(), mag + add.double().abs()
            _within(dx, want, mag, K + 1)
            if dw is not None:
                want, mag = plain.dots(x.double(), finite, slot)
                _within(dw, want, mag, H, half=0.0)
    dx2 = add.cuda().clone()                                      # added in place
    ep.ep_sort_backward(td, s, dx2, weights=wd, add=dx2)
    assert torch.equal(dx2, ep.ep_sort_backward(td, s, torch.empty_like(dx2), weights=wd, add=add.cuda()))
    alone = torch.empty(T, K, device="cuda")                      # the weights' gradient alone
    ep.ep_sort_backward(td, s, weights=wd, x=xd, d_weights=alone)
    both = torch.empty_like(alone)
    ep.ep_sort_backward(td, s, dx2, weights=wd, x=xd, d_weights=both)
    assert torch.equal(alone, both) and int(status) == 0


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("T,K,H", SHAPES)
@pytest.mark.parametrize("p", [0.0, 0.3])
def test_combine_and_its_gradients(T, K, H, p, shared):
    slot, w, out, dy, res, named = _data(T, K, H, 3 * T + K + H, shared=shared)
    rows, s, od, dyd, wd = out.shape[0], slot.int().cuda(), out.cuda(), dy.cuda(), w.cuda()
    w64 = torch.where(slot >= 0, w.double(), 0.0)
    seed, step, site = 0x123456789ABCDEF - T, (1 << 32) + 7, 0xFFFFFFF0
    drop = ep.Dropout(p, torch.tensor([seed, step], device="cuda"), site) if p else None
    k = plain.keep(T, H, p, seed, step, site)
    finite = torch.where(named[:, None], out.double(), 0.0)
    want, mag = plain.gather(finite, slot, w64)
    want, mag = want * k, mag * k
    y = ep.ep_combine_residual(od, s, wd, torch.empty(T, H, dtype=BF, device="cuda"), dropout=drop)
    _within(y, want, mag, K)
    if not p:
        assert torch.equal(y, ep.ep_combine(od, s, wd, torch.empty_like(y), 1, 1))
    y = res.cuda().clone()
    ep.ep_combine_residual(od, s, wd, y, residual=y, dropout=drop)                 # in place
    _within(y, want + res.double(), mag + res.double().abs(), K + 1)

    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    whole, d_out = guarded(rows, H)
    before, dw = d_out.clone(), torch.full((T, K), 9.0, device="cuda")
    ep.ep_combine_backward(dyd, s, wd, d_out, out=od, d_weights=dw, dropout=drop, status=status)
    g = dy.double() * k
    want, _ = plain.spread(g, slot, w64, rows)
    mag, _ = plain.spread(g.abs(), slot, w64, rows)
    _within(d_out[named.cuda()], want[named], mag[named], K)
    assert torch.equal(d_out[~named.cuda()].view(torch.int16), before[~named.cuda()].view(torch.int16)) and guards_intact(whole)
    want, mag = plain.dots(g, finite, slot)
    _within(dw, want, mag, H, half=0.0)
    alone = torch.empty_like(dw)
    ep.ep_combine_backward(dyd, s, wd, out=od, d_weights=alone, dropout=drop)      # either alone, and in place of out
    rows_alone = torch.zeros_like(od)
    ep.ep_combine_backward(dyd, s, wd, rows_alone, dropout=drop)
    same = od.clone()
    ep.ep_combine_backward(dyd, s, wd, same, out=same, d_weights=dw, dropout=drop)
    m = named.cuda()
    assert torch.equal(alone, dw) and torch.equal(rows_alone[m], d_out[m]) and torch.equal(same[m], d_out[m]) and int(status) == 0


def test_slots_past_the_buffer_are_skipped():
    T, K, H, rows = 6, 2, 64, 5
    slot = torch.arange(T * K, dtype=torch.int32, device="cuda").view(T, K)
    x, w = torch.ones(T, H, dtype=BF, device="cuda"), torch.full((T, K), 0.5, device="cuda")
    for call in (lambda st, buf, d: ep.ep_sort(x, slot, buf, weights=w, status=st),
                 lambda st, buf, d: ep.ep_combine_backward(x, slot, w, buf, out=buf, d_weights=d, status=st),
                 lambda st, buf, d: ep.ep_sort_backward(buf, slot, torch.empty_like(x), weights=w, x=x, d_weights=d, status=st)):
        whole, buf = guarded(rows, H)
        buf.fill_(1.0)
        st, d = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(T, K, device="cuda")
        call(st, buf, d)
        assert int(st) == ep.STATUS_CAPACITY and guards_intact(whole) and torch.isfinite(buf).all()
        assert (d.flatten()[rows:] == 0).all()


def test_no_tokens_is_no_work():
    e = torch.empty(0, 64, dtype=BF, device="cuda")
    s, w, rows = torch.empty(0, 2, dtype=torch.int32, device="cuda"), torch.empty(0, 2, device="cuda"), torch.ones(4, 64, dtype=BF, device="cuda")
    ep.ep_sort(e, s, rows, weights=w)
    ep.ep_sort_backward(rows, s, e, weights=w)
    ep.ep_combine_residual(rows, s, w, e)
    ep.ep_combine_backward(e, s, w, rows)
    assert (rows == 1).all()
    ep.ep_dropout(e, ep.Dropout(0.5, torch.zeros(2, dtype=torch.int64, device="cuda")), y=e)


@pytest.mark.parametrize("rows,cols,limit", [(1, 8, None), (3, 24, 2), (257, 264, 200), (1000, 1032, 0), (64, 4096, 64), (129, 2048, 1000)])
@pytest.mark.parametrize("p", [0.1, 0.5, 1.0, 1e-6])
def test_dropout(rows, cols, limit, p):
    g = torch.Generator().manual_seed(rows + cols)
    x, res = (torch.randn(rows, cols, generator=g).to(BF) for _ in range(2))
    seed, step, site = -5, 3, 9
    drop = ep.Dropout(p, torch.tensor([seed, step], device="cuda"), site)
    k = plain.keep(rows, cols, p, seed % (1 << 64), step, site)
    x[k == 0] = float("inf")                                     # what is dropped does not matter
    x[0, 0] = float("nan") if float(k[0, 0]) == 0 else x[0, 0]
    n = rows if limit is None else min(rows, limit)
    lim = None if limit is None else torch.tensor([limit], dtype=torch.int32, device="cuda")
    clean = torch.where(k == 0, 0.0, x.double())
    for residual in (None, res):
        whole, y = guarded(rows, cols)
        before = y.clone()
        ep.ep_dropout(x.cuda(), drop, residual=None if residual is None else residual.cuda(), y=y, limit=lim)
        want = clean * k + (0.0 if residual is None else res.double())
        mag = (clean * k).abs() + (0.0 if residual is None else res.double().abs())
        _within(y[:n], want[:n], mag[:n], 2)
        assert torch.equal(y[n:].view(torch.int16), before[n:].view(torch.int16)) and guards_intact(whole)
    y = x.cuda()
    ep.ep_dropout(y, drop, residual=y, y=y)                       # all three one buffer
    want = ep.ep_dropout(x.cuda(), drop, residual=x.cuda())
    assert torch.equal(y.view(torch.int16), want.view(torch.int16))


def test_dropout_in_a_graph_takes_the_state_of_the_replay():
    x = torch.randn(64, 256, device="cuda").to(BF)
    state = torch.tensor([11, 0], device="cuda")
    drop, y = ep.Dropout(0.5, state), torch.empty_like(x)
    ep.ep_dropout(x, drop, y=y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ep.ep_dropout(x, drop, y=y)
        state[1] += 1
    for step in range(3):
        graph.replay()
        assert torch.equal(y, ep.ep_dropout(x, ep.Dropout(0.5, torch.tensor([11, step], device="cuda"))))
