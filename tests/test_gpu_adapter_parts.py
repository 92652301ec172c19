"""The adapters' gradients where long adapters are cut and their parts added: beside short and empty ones, at ranks of one and two chunks, with and
without an index, many times over, on two streams at once and from a graph. Tolerances as in test_gpu_adapters.py."""
import pytest
import torch

import train_plain as plain
from adapter_plan import parts
from paper_2609_40093_b200 import ep
from test_gpu_adapters import _abs_terms, _within

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
BESIDE = [0, 3, 700, 0, 64, 4100, 65, 0] + [1] * 20                   # what lies beside an adapter of 15000 entries
LONG = [  # rows, H, N, rank, entries of each adapter, mixed, parts of the combined call
    (16384, 64, 72, 16, [16384], False, 16), (32000, 136, 64, 64, [31000, 0], True, 16), (20000, 128, 72, 8, [15000] + BESIDE, True, 16),
    (20000, 136, 200, 104, BESIDE + [14000], False, 12), (9000, 264, 200, 24, [9000], True, 8), (24000, 64, 200, 72, [9000, 8000, 7000], True, 8),
    (24000, 64, 200, 32, [9000, 8000, 7000], False, 8), (5000, 72, 264, 128, [0, 4993], False, 6),
]


def _offsets(counts):
    return torch.cat([torch.zeros(1, dtype=torch.long), torch.cumsum(torch.tensor(counts), 0)])


def _problem(rows, H, N, r, counts, mixed, seed):
    g, A = torch.Generator().manual_seed(seed), len(counts)
    index = torch.randperm(rows, generator=g) if mixed else None
    c = {k: torch.randn(rows, n, generator=g).to(BF) for k, n in (("x", H), ("dy", N), ("base", N), ("dbase", H), ("mid", r))}
    c.update(down=(torch.randn(A, r, H, generator=g) * H ** -0.5).to(BF), up=(torch.randn(A, N, r, generator=g) * r ** -0.5).to(BF),
             scale=torch.rand(A, generator=g) + 0.5, offsets=_offsets(counts), index=index)
    d = {k: v.cuda() for k, v in c.items() if k not in ("offsets", "index")}
    d.update(off=c["offsets"].int().cuda(), index=None if index is None else index.int().cuda(), adapters=ep.Adapters(d["down"], d["up"], d["scale"]))
    return c, d


def _backward(d, grads, status=None):
    grads.workspace.fill_(0xFF)                                       # NaN, were it used before it is written
    return ep.ep_adapter_matmul_backward(d["dy"], d["x"], d["off"], d["adapters"], d["mid"], grads, base=d["dbase"] if grads.dx is not None else None,
                                         row_index=d["index"], status=status)


@pytest.mark.parametrize("case", LONG, ids=lambda c: "-".join(str(v) for v in c[:4]) + ("-mixed" if c[5] else ""))
def test_parts_are_added_right_and_the_same_every_time(case):
    rows, H, N, r, counts, mixed, most = case
    c, d = _problem(rows, H, N, r, counts, mixed, rows + H + r)
    assert max(parts(c["offsets"], rows, H, N, r)) == most
    n, z = int(c["offsets"][-1]), {k: c[k].double() for k in ("dy", "x", "dbase", "down", "up", "scale", "mid")}
    z["mid"][n:] = 0
    want = dict(zip(("dx", "ddown", "dup"), plain.adapter_grads(z["dy"], z["x"], z["dbase"], c["offsets"], c["index"], z["down"], z["up"], z["scale"], z["mid"])))
    err = _abs_terms(c, z["mid"])
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    first = ep.alloc_adapter_grads(d["x"], d["adapters"], entries=rows)
    first.dx.copy_(d["dbase"])
    _backward(d, first, status)
    assert int(status) == 0
    for name, w in want.items():
        _within(getattr(first, name), w, err[name])
    again = ep.alloc_adapter_grads(d["x"], d["adapters"], entries=rows)
    again.dx.copy_(d["dbase"])
    for _ in range(20):
        again.ddown.fill_(float("nan")), again.dup.fill_(float("nan"))
        _backward(d, again)
        assert all(torch.equal(getattr(again, k), getattr(first, k)) for k in want)
    for name in ("ddown", "dup"):                                     # one alone is cut in other places
        one = ep.alloc_adapter_grads(d["x"], d["adapters"], entries=rows, dx=False, down=name == "ddown", up=name == "dup")
        _within(getattr(_backward(d, one), name), want[name], err[name])


def test_parts_on_two_streams_and_from_a_graph():
    cases = [(20000, 128, 72, 64, [15000] + BESIDE, True), (16384, 136, 72, 40, [9000, 7000], False)]
    made = [_problem(*c, seed=i) for i, c in enumerate(cases)]
    assert all(max(parts(c["offsets"], *case[:4])) > 4 for (c, _), case in zip(made, cases))
    want, got = [], []
    for _, d in made:
        for keep in (want, got):
            keep.append(ep.alloc_adapter_grads(d["x"], d["adapters"]))
            keep[-1].dx.copy_(d["dbase"])
        _backward(d, want[-1])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in made]
    for _ in range(10):
        for s, (_, d), g in zip(streams, made, got):
            with torch.cuda.stream(s):
                _backward(d, g)
    torch.cuda.synchronize()

    def equal():
        return all(torch.equal(getattr(g, k), getattr(w, k)) for g, w in zip(got, want) for k in ("dx", "ddown", "dup"))

    assert equal()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for (_, d), g in zip(made, got):
            _backward(d, g)
    for _ in range(10):
        for g in got:
            g.ddown.zero_(), g.dup.zero_()
        graph.replay()
        assert equal()
