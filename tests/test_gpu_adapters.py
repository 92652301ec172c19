"""ep_adapter_matmul and its gradients against their plain statements in 64 bits.

Tolerances, element by element: the tensor cores' fp32 sums of n exact products are off by at most n 2^-23 of the sum of their magnitudes
(they may truncate where an fp32 addition rounds); mid and dmid are then rounded to bf16 (2^-8), which reaches the second product through the
magnitudes of its weights; the result is rounded once more."""
import pytest
import torch

import train_plain as plain
from gpu_util import guarded, guards_intact
from paper_2609_40093_b200 import ep

pytestmark = pytest.mark.gpu
BF, HALF = torch.bfloat16, 2.0 ** -8


def _sum(n):
    return (n + 4) * 2.0 ** -23


def _counts(kind, n, A, g):
    if kind == "one":
        c = torch.zeros(A, dtype=torch.long)
        c[A // 2] = n
    elif kind == "spread":
        c = torch.full((A,), n // A)
        c[:n % A] += 1
    else:                                                        # a few with many, most with few or none
        c = torch.bincount(torch.randint(0, A, (n,), generator=g) * torch.randint(0, 2, (n,), generator=g), minlength=A)
    return c


def _case(rows, H, N, r, A, kind, mixed, without, seed):
    g = torch.Generator().manual_seed(seed)
    n = rows - int(rows * without)
    offsets = torch.cat([torch.zeros(1, dtype=torch.long), torch.cumsum(_counts(kind, n, A, g), 0)])
    index = torch.randperm(rows, generator=g) if mixed else None
    x, dy, base, dbase = (torch.randn(rows, c, generator=g).to(BF) for c in (H, N, N, H))
    down, up = (torch.randn(A, r, H, generator=g) * H ** -0.5).to(BF), (torch.randn(A, N, r, generator=g) * r ** -0.5).to(BF)
    scale = torch.rand(A, generator=g) + 0.5
    named = torch.zeros(rows, dtype=torch.bool)
    named[index[:n] if mixed else slice(0, n)] = True
    x[~named], dy[~named] = float("nan"), float("nan")           # rows without an adapter take no part, whatever they hold
    return dict(n=n, rows=rows, offsets=offsets, index=index, x=x, dy=dy, base=base, dbase=dbase, down=down, up=up, scale=scale, named=named)


def _abs_terms(c, mid):
    """Sums of magnitudes behind mid, y, dmid, dx, ddown, dup."""
    z = {k: c[k].double().abs() for k in ("x", "dy", "down", "up", "scale")}
    out = {"mid": torch.zeros_like(mid), "y": torch.zeros(c["base"].shape, dtype=torch.float64), "dmid": torch.zeros_like(mid),
           "dx": torch.zeros(c["dbase"].shape, dtype=torch.float64), "ddown": torch.zeros(c["down"].shape, dtype=torch.float64),
           "dup": torch.zeros(c["up"].shape, dtype=torch.float64)}
    H, N, r = c["x"].shape[1], c["dy"].shape[1], mid.shape[1]
    for a, e, row in plain.entries(c["offsets"], c["index"]):
        x, dy, down, up, s = z["x"][row], z["dy"][row], z["down"][a], z["up"][a], z["scale"][a]
        m_mag, g_mag = x @ down.t(), s * (dy @ up)
        m_err = _sum(H) * m_mag + HALF * (mid[e].abs() + _sum(H) * m_mag)
        dmid = (s * (c["dy"][row].double() @ c["up"][a].double())).abs()
        g_err = _sum(N) * g_mag + HALF * (dmid + _sum(N) * g_mag)
        out["mid"][e], out["dmid"][e] = m_err, g_err
        out["y"][row] = s * (m_err @ up.t()) + _sum(r) * s * ((mid[e].abs() + m_err) @ up.t())
        out["dx"][row] = g_err @ down + _sum(r) * ((dmid + g_err) @ down)
        out["ddown"][a] = g_err.t() @ x + _sum(len(e)) * ((dmid + g_err).t() @ x)
        out["dup"][a] = _sum(len(e)) * s * (dy.t() @ mid[e].abs())
    return out


def _within(got, want, err):
    got = got.double().cpu()
    bad = ~((got - want).abs() <= HALF * (want.abs() + err) + err + 2.0 ** -133)
    assert not bad.any(), (int(bad.sum()), bad.numel(), float((got - want).abs().max()), float(err.max()))


CASES = [  # rows, H, N, r, A, distribution, mixed, share without
    (1, 64, 64, 8, 1, "one", False, 0.0), (1, 4096, 512, 16, 32, "one", True, 0.0), (2, 72, 136, 8, 3, "spread", True, 0.0),
    (5, 520, 264, 24, 4, "few", True, 0.0), (64, 1024, 1032, 16, 64, "spread", True, 0.0), (256, 512, 768, 16, 40, "few", True, 0.1),
    (130, 200, 8, 128, 2, "one", False, 0.0), (128, 8, 200, 64, 1, "one", False, 0.0), (129, 2048, 384, 72, 5, "few", False, 0.2),
    (700, 264, 520, 40, 3, "few", True, 0.3), (1003, 520, 264, 24, 12, "few", True, 0.1), (1500, 4096, 128, 128, 1, "one", True, 0.0),
    (2000, 128, 2048, 32, 300, "few", False, 0.0), (300, 1024, 1024, 112, 2, "spread", True, 0.0), (3000, 768, 640, 64, 2, "spread", False, 0.0),
    (40, 640, 640, 8, 4096, "few", True, 0.5), (50, 1024, 1544, 32, 1, "one", True, 0.0), (64, 136, 2056, 128, 1, "one", False, 0.0),
    (190, 2048, 520, 24, 4, "spread", True, 0.0), (33, 4096, 136, 16, 1, "one", False, 0.0),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(v) for v in c))
def test_forward_and_gradients(case):
    rows, H, N, r, A, kind, mixed, without = case
    c = _case(rows, H, N, r, A, kind, mixed, without, sum(case[:5]))
    named, off = c["named"], c["offsets"].int().cuda()
    finite = {k: torch.where(named[:, None], c[k].double(), 0.0) for k in ("x", "dy")}
    mid64, y64 = plain.adapters(finite["x"], c["base"].double(), c["offsets"], c["index"], c["down"].double(), c["up"].double(), c["scale"].double(), rows)
    err = _abs_terms(dict(c, **finite), mid64)
    d = {k: c[k].cuda() for k in ("x", "dy", "base", "dbase", "down", "up", "scale")}
    index = None if c["index"] is None else c["index"].int().cuda()
    ad, status = ep.Adapters(d["down"], d["up"], d["scale"]), torch.zeros(1, dtype=torch.int32, device="cuda")
    whole, y = guarded(rows, N)
    y.copy_(d["base"])
    whole_mid, mid = guarded(rows, r)
    before = mid.clone()
    ep.ep_adapter_matmul(d["x"], off, ad, y, base=d["base"], row_index=index, mid=mid, status=status)
    assert int(status) == 0 and guards_intact(whole) and guards_intact(whole_mid)
    assert torch.equal(y[~named.cuda()], d["base"][~named.cuda()]) and torch.equal(mid[c["n"]:].view(torch.int16), before[c["n"]:].view(torch.int16))
    _within(mid[:c["n"]], mid64[:c["n"]], err["mid"][:c["n"]])
    _within(y, y64, err["y"])
    again = d["base"].clone()                                     # in place, without mid: the same bits
    ep.ep_adapter_matmul(d["x"], off, ad, again, base=again, row_index=index)
    assert torch.equal(again, y)
    delta = torch.zeros_like(d["base"])                           # nothing to add to
    ep.ep_adapter_matmul(d["x"], off, ad, delta, row_index=index)
    _within(delta[named.cuda()], (y64 - c["base"].double())[named], err["y"][named])
    only = torch.zeros_like(mid)                                  # the first product alone
    ep.ep_adapter_matmul(d["x"], off, ad, mid=only, row_index=index)
    assert torch.equal(only[:c["n"]], mid[:c["n"]])

    # gradients, from the mid that was written
    seen = mid.double().cpu()
    seen[c["n"]:] = 0
    want = plain.adapter_grads(finite["dy"], finite["x"], c["dbase"].double(), c["offsets"], c["index"], c["down"].double(), c["up"].double(),
                               c["scale"].double(), seen)
    err = _abs_terms(dict(c, **finite), seen)
    grads = ep.alloc_adapter_grads(d["x"], ad, entries=rows)
    guard = {}
    for name in ("dx", "ddown", "dup"):
        t = getattr(grads, name)
        guard[name], inner = guarded(t.numel() // t.shape[-1], t.shape[-1])
        setattr(grads, name, inner.view(t.shape))
    grads.dx.copy_(d["dbase"])
    grads.workspace.fill_(0xFF)                                   # NaN, were it used before it is written
    ep.ep_adapter_matmul_backward(d["dy"], d["x"], off, ad, mid, grads, base=d["dbase"], row_index=index, status=status)
    assert int(status) == 0 and all(guards_intact(w) for w in guard.values())
    for name, w in zip(("dx", "ddown", "dup"), want):
        _within(getattr(grads, name), w, err[name])
    # the same call gives the same bits; each gradient alone may be summed in other parts
    again = ep.alloc_adapter_grads(d["x"], ad, entries=rows)
    again.dx.copy_(d["dbase"])
    ep.ep_adapter_matmul_backward(d["dy"], d["x"], off, ad, mid, again, base=d["dbase"], row_index=index)
    assert all(torch.equal(getattr(again, name), getattr(grads, name)) for name in ("dx", "ddown", "dup"))
    for name, w in zip(("dx", "ddown", "dup"), want):
        one = ep.alloc_adapter_grads(d["x"], ad, entries=rows, dx=name == "dx", down=name == "ddown", up=name == "dup")
        if name == "dx":
            one.dx.copy_(d["dbase"])
        ep.ep_adapter_matmul_backward(d["dy"], d["x"], off, ad, mid, one, base=one.dx, row_index=index)
        _within(getattr(one, name), w, err[name])
        assert name != "dx" or torch.equal(one.dx, grads.dx)


def test_adapters_laid_out_by_the_library():
    """ids [T] of a decode batch, -1 for none, through ep_layout with one pick and one rank."""
    g = torch.Generator().manual_seed(5)
    T, H, N, r, A = 96, 256, 320, 16, 10
    ids = torch.randint(-1, A, (T,), generator=g)
    lay = ep.ep_layout(ids.int().view(T, 1).cuda(), A, 1)
    x, base = torch.randn(T, H, generator=g).to(BF), torch.randn(T, N, generator=g).to(BF)
    down, up = (torch.randn(A, r, H, generator=g) / 16).to(BF), (torch.randn(A, N, r, generator=g) / 4).to(BF)
    y = base.cuda()
    ep.ep_adapter_matmul(x.cuda(), lay.expert_offsets, ep.Adapters(down.cuda(), up.cuda()), y, base=y, row_index=lay.pair_token)
    want = base.double()
    for t in range(T):
        if ids[t] >= 0:
            want[t] += up[ids[t]].double() @ (down[ids[t]].double() @ x[t].double())
    err = (y.double().cpu() - want).norm() / want.norm()
    assert float(err) < 2 * HALF and torch.equal(y.cpu()[ids < 0], base[ids < 0])


def test_offsets_and_rows_out_of_range():
    T, H, N, r, A = 20, 64, 64, 8, 2
    g = torch.Generator().manual_seed(6)
    x, dy = (torch.randn(T, H, generator=g).to(BF).cuda() for _ in range(2))
    ad = ep.Adapters((torch.randn(A, r, H, generator=g) / 8).to(BF).cuda(), torch.randn(A, N, r, generator=g).to(BF).cuda())
    index = torch.arange(T, dtype=torch.int32, device="cuda")
    index[3], index[15] = T, -1                                   # rows that do not exist
    off = torch.tensor([0, 10, T + 50], dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    whole, y = guarded(T, N)
    y.zero_()
    mid = torch.full((T, r), 9.0, dtype=BF, device="cuda")
    ep.ep_adapter_matmul(x, off, ad, y, row_index=index, mid=mid, status=status)
    assert int(status) == (ep.STATUS_CAPACITY | ep.STATUS_BAD_INDEX) and guards_intact(whole)
    good = [i for i in range(T) if i not in (3, 15)]
    assert (mid[[3, 15]] == 0).all() and (y[[3, 15]] == 0).all() and (y[good].abs().sum(1) > 0).all()
    status.zero_()
    grads = ep.alloc_adapter_grads(x, ad)
    mid[[3, 15]] = float("nan")                                   # entries without a row take no part
    ep.ep_adapter_matmul_backward(dy, x, off, ad, mid, grads, row_index=index, status=status)
    assert int(status) & ep.STATUS_BAD_INDEX and torch.isfinite(grads.ddown).all() and torch.isfinite(grads.dup).all()
    mid[[3, 15]] = 0
    want = plain.adapter_grads(dy.double().cpu(), x.double().cpu(), torch.zeros(T, H, dtype=torch.float64), [0, 9, 18],
                               torch.tensor(good), ad.down.double().cpu(), ad.up.double().cpu(), torch.ones(A), mid[good].double().cpu())
    assert float((grads.dup.double().cpu() - want[2]).norm() / want[2].norm()) < HALF
    assert float((grads.ddown.double().cpu() - want[1]).norm() / want[1].norm()) < 2 * HALF


def test_offsets_that_decrease_are_refused_on_the_device():
    """They name every entry many times over: more pieces than the workspace has room for."""
    T, H, N, r, A = 3000, 64, 64, 8, 64
    x = torch.randn(T, H, device="cuda").to(BF)
    ad = ep.Adapters((torch.randn(A, r, H, device="cuda") / 8).to(BF), torch.randn(A, N, r, device="cuda").to(BF))
    off = torch.tensor([T * (i % 2) for i in range(A + 1)], dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    mid, grads = torch.zeros(T, r, dtype=BF, device="cuda"), ep.alloc_adapter_grads(x, ad)
    ws = torch.full((grads.workspace.numel() + 512,), 0x5A, dtype=torch.uint8, device="cuda")
    grads.workspace, grads.ddown, grads.dup = ws[256:-256], grads.ddown.fill_(3.0), grads.dup.fill_(3.0)
    for dx in (grads.dx, None):
        grads.dx = dx
        status.zero_()
        ep.ep_adapter_matmul_backward(x, x, off, ad, mid, grads, status=status)
        assert int(status) == ep.STATUS_CAPACITY and (grads.ddown == 3).all() and (grads.dup == 3).all()
        assert (ws[:256] == 0x5A).all() and (ws[-256:] == 0x5A).all()


def test_no_entries():
    T, H, N, r, A = 4, 64, 64, 8, 3
    x = torch.ones(T, H, dtype=BF, device="cuda")
    ad = ep.Adapters(torch.ones(A, r, H, dtype=BF, device="cuda"), torch.ones(A, N, r, dtype=BF, device="cuda"))
    y = torch.full((T, N), 5.0, dtype=BF, device="cuda")
    off = torch.zeros(A + 1, dtype=torch.int32, device="cuda")
    empty = torch.empty(0, dtype=torch.int32, device="cuda")
    for index in (None, empty):
        ep.ep_adapter_matmul(x, off, ad, y, base=y, row_index=index)
        grads = ep.alloc_adapter_grads(x, ad)
        grads.dx.fill_(3.0)
        ep.ep_adapter_matmul_backward(y, x, off, ad, torch.zeros(T if index is None else 0, r, dtype=BF, device="cuda"), grads, base=grads.dx, row_index=index)
        assert (y == 5).all() and (grads.dx == 3).all() and (grads.ddown == 0).all() and (grads.dup == 0).all()
