"""ep_adapter_matmul and its gradients with an infinite element in a row that an adapter has: the definition's infinities come out, at ranks
that fill the tensor cores' steps of 16 and at ranks that do not, and nothing else changes by a bit.

Signs are laid out so that no sum meets infinities of both signs: `up` has the sign of its output feature's parity, `down` that of its input
feature's. Nothing is compared by a tolerance: infinities have a place and a sign, all else is the bits of the call without them."""
import pytest
import torch

from paper_2609_40093_b200 import ep

pytestmark = pytest.mark.gpu
BF, INF = torch.bfloat16, float("inf")


def _run(x, dy, off, ad, index, base, dbase):
    rows, r = x.shape[0], ad.down.shape[1]
    y, mid = base.clone(), torch.zeros(rows, r, dtype=BF, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ep.ep_adapter_matmul(x, off, ad, y, base=base, row_index=index, mid=mid, status=status)
    grads = ep.alloc_adapter_grads(x, ad, entries=rows)
    grads.dx.copy_(dbase)
    ep.ep_adapter_matmul_backward(dy, x, off, ad, mid, grads, base=dbase, row_index=index, status=status)
    assert int(status) == 0
    return {k: v.cpu() for k, v in dict(y=y, mid=mid, dx=grads.dx, ddown=grads.ddown, dup=grads.dup).items()}


@pytest.mark.parametrize("rows,H,N,r,A,mixed", [
    (3, 4096, 136, 8, 2, True), (40, 64, 64, 16, 2, False), (200, 4096, 264, 24, 2, False), (700, 72, 136, 8, 3, True), (700, 264, 520, 40, 3, False),
    (130, 200, 72, 72, 2, False), (130, 200, 72, 104, 2, True), (64, 512, 2056, 64, 4, True)])
def test_an_infinite_element_gives_the_definitions_infinities(rows, H, N, r, A, mixed):
    g = torch.Generator().manual_seed(rows + H + r)

    def far_from_zero(*shape):
        t = torch.randn(*shape, generator=g)
        return torch.where(t < 0, t - 0.1, t + 0.1)

    def parity(n):
        return 1.0 - 2.0 * (torch.arange(n) % 2)

    x, dy, base, dbase = (far_from_zero(rows, c).to(BF).cuda() for c in (H, N, N, H))
    down = (far_from_zero(A, r, H).abs() * parity(H) * H ** -0.5).to(BF).cuda()
    up = (far_from_zero(A, N, r).abs() * parity(N)[:, None] * r ** -0.5).to(BF).cuda()
    ad = ep.Adapters(down, up, torch.rand(A, generator=g).cuda() + 0.5)
    cut = [rows * a // A for a in range(A + 1)]
    off = torch.tensor(cut, dtype=torch.int32, device="cuda")
    index = torch.randperm(rows, generator=g).int().cuda() if mixed else None
    place = torch.arange(rows) if index is None else index.cpu().long()
    e0, e1 = cut[1] - 1, cut[2] - 1                                  # the last entries of adapters 0 and 1
    r0, r1 = int(place[e0]), int(place[e1])
    want = _run(x, dy, off, ad, index, base, dbase)
    assert all(torch.isfinite(v.float()).all() for v in want.values())
    f = H - 2                                                        # even: down is positive there
    x[r0, f], dy[r1, 0] = INF, INF
    got = _run(x, dy, off, ad, index, base, dbase)

    want["y"][r0] = INF * parity(N).to(BF)                           # mid is infinite throughout
    want["mid"][e0] = INF
    want["dx"][r1] = INF * parity(H).to(BF)                          # dmid is
    want["ddown"][0, :, f] = got["ddown"][0, :, f]                   # dmid of row r0 times infinity: its sign is dmid's
    assert torch.isinf(got["ddown"][0, :, f].float()).all()
    want["ddown"][1] = (INF * x[r1].sign()).cpu()                    # an infinite dmid times the row
    want["dup"][0] = (INF * dy[r0].sign()).cpu()[:, None]            # the row of dy times an infinite mid
    want["dup"][1, 0] = (INF * got["mid"][e1].float().sign()).to(BF)
    for name in got:
        assert torch.equal(got[name].float(), want[name].float()), (name, int((got[name].float() != want[name].float()).sum()))
