"""The experts' products and their gradients on the GPU against the 64-bit statements of `moe_plain`.

Tolerances, from the number formats: products of bf16 are exact in fp32; a sum of n of them errs by at most n 2^-23 of the
sum S of their absolute values (each addition may truncate); the activations are 1.13-Lipschitz and their own fp32 error is
below 2^-18 (1 + |z|); the result is rounded once to bf16, 2^-8 relative covers half an ulp. dz is rounded to bf16 in front
of the gradient's products (2^-9 of S at most, 2^-8 with the error of the slope)."""
import math

import pytest
import torch

import moe_plain as plain
from paper_2609_40093_b200 import ep

pytestmark = pytest.mark.gpu

ACTS = {"none": ep.ACT_NONE, "relu": ep.ACT_RELU, "silu": ep.ACT_SILU, "gelu": ep.ACT_GELU}


def _case(counts, H, N, seed=0, slack=0):
    """x and dy (with `slack` rows of NaN behind the segments), offsets, weight, bias, operand."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def mk(*shape, scale=1.0):
        return (torch.randn(*shape, device="cuda", generator=g) * scale).bfloat16()

    E, P = len(counts), sum(counts)
    off = torch.tensor([0] + list(torch.tensor(counts).cumsum(0)), dtype=torch.int32, device="cuda")
    c = dict(x=mk(P + slack, H), offsets=off, weight=mk(E, N, H, scale=H ** -0.5), bias=mk(E, N, scale=0.5), operand=mk(P + slack, N),
             dy=mk(P + slack, N), P=P)
    for k in ("x", "operand", "dy"):
        c[k][P:] = math.nan
    return c


def _guarded(rows, cols):
    whole = torch.full((rows + 2, cols), 31.0, dtype=torch.bfloat16, device="cuda")
    return whole, whole[1:-1]


def _check_forward(c, name="none", bias=False, op="none", pre=False):
    P, (E, N, H) = c["P"], c["weight"].shape
    rows = c["x"].shape[0]
    whole, y = _guarded(rows, N)
    wpre, z_out = _guarded(rows, N)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    b, r = (c["bias"] if bias else None), (c["operand"] if op != "none" else None)
    ep.ep_expert_matmul(c["x"], c["offsets"], c["weight"], bias=b, activation=ACTS[name], operand=r,
                        operand_op=ep.OPERAND_MUL if op == "mul" else ep.OPERAND_ADD, y=y, pre=z_out if pre else None, status=status)
    want, z, S = plain.experts(c["x"], c["offsets"], c["weight"], b, name, r, op == "mul")
    zerr = (H + 1) * 2.0 ** -23 * S
    factor = r[:P].double().abs() if op == "mul" else 1.0
    tol = 2.0 ** -8 * want.abs() + factor * (1.13 * zerr + 2.0 ** -18 * (1 + z.abs())) + 1e-30
    err = (y[:P].double() - want).abs()
    assert (err <= tol).all(), (float((err - tol).max()), torch.nonzero(err > tol)[:4].tolist())
    assert (whole[0] == 31).all() and (whole[1 + P:] == 31).all()                 # nothing outside the segments' rows
    if pre:
        assert ((z_out[:P].double() - z).abs() <= 2.0 ** -8 * z.abs() + zerr).all()
        assert (wpre[0] == 31).all() and (wpre[1 + P:] == 31).all()
    assert int(status) == 0
    return y


COUNTS = [[1], [0], [0, 1, 0], [64], [16, 17, 15], [1] * 40, [100, 0, 3, 64, 65, 1], [300], [513, 2, 255, 256, 257], [0, 0, 700, 0]]


@pytest.mark.parametrize("counts", COUNTS, ids=str)
@pytest.mark.parametrize("H,N", [(64, 128), (8, 8), (72, 136), (520, 264), (1024, 96)])
def test_products_of_ragged_segments(counts, H, N):
    c = _case(counts, H, N, seed=sum(counts) + H)
    if c["P"]:
        _check_forward(c)


@pytest.mark.parametrize("name", list(ACTS))
@pytest.mark.parametrize("op", ["none", "add", "mul"])
@pytest.mark.parametrize("bias", [False, True])
def test_epilogues(name, op, bias):
    for counts in ([70, 0, 5], [600, 40]):
        _check_forward(_case(counts, 136, 200, slack=9), name, bias, op, pre=True)


def test_rows_behind_the_segments_and_other_experts_nan_stay_out():
    """NaN in the slack rows, and in one expert's rows or weights, reaches neither other experts' results nor their gradients."""
    counts, H, N = [37, 70, 21], 200, 136
    c = _case(counts, H, N, slack=50)
    c["x"][37:107] = math.nan                                   # expert 1's rows
    y = ep.ep_expert_matmul(c["x"], c["offsets"], c["weight"])
    assert torch.isfinite(y[:37]).all() and torch.isfinite(y[107:128]).all() and torch.isnan(y[37:107]).all()
    c["dy"][37:107] = math.inf
    g = ep.ep_expert_matmul_backward(c["dy"], c["x"], c["offsets"], c["weight"],
                                     grads=ep.alloc_expert_grads(c["x"].shape[0], H, N, 3, bias=True))
    assert torch.isfinite(g.dx[:37]).all() and torch.isfinite(g.dx[107:128]).all()
    for e in (0, 2):
        assert torch.isfinite(g.dweight[e]).all() and torch.isfinite(g.dbias[e]).all()
    assert not torch.isfinite(g.dweight[1]).any()
    c = _case(counts, H, N)
    c["weight"][1] = math.nan
    y = ep.ep_expert_matmul(c["x"], c["offsets"], c["weight"])
    assert torch.isfinite(y[:37]).all() and torch.isfinite(y[107:]).all()


def _check_backward(c, name="none", op="none", wanted=("dx", "dweight", "dbias", "doperand"), poison=True):
    P, (E, N, H) = c["P"], c["weight"].shape
    rows = c["x"].shape[0]
    g = torch.Generator(device="cuda").manual_seed(9)
    pre = torch.randn(rows, N, device="cuda", generator=g).bfloat16() * 1.5
    pre[P:] = math.nan
    mul = op == "mul"
    grads = ep.alloc_expert_grads(rows, H, N, E, x="dx" in wanted, weight="dweight" in wanted, bias="dbias" in wanted,
                                  operand=mul and "doperand" in wanted)
    if poison:
        grads.workspace.fill_(255)                              # NaN in every fp32 and bf16 word
        for t in (grads.dweight, grads.dbias):
            if t is not None:
                t.fill_(math.nan)
    wdx, dx = _guarded(rows, H)
    wdo, dop = _guarded(rows, N)
    if grads.dx is not None:
        grads.dx = dx
    if grads.doperand is not None:
        grads.doperand = dop
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ep.ep_expert_matmul_backward(c["dy"], c["x"], c["offsets"], c["weight"], pre=pre if name != "none" or mul else None, activation=ACTS[name],
                                 operand=c["operand"] if op != "none" else None,
                                 operand_op=ep.OPERAND_MUL if mul else ep.OPERAND_ADD, grads=grads, status=status)
    want, size = plain.experts_gradient(c["dy"], c["x"], c["offsets"], c["weight"], pre, name, c["operand"], mul)
    longest = max(1, int((c["offsets"][1:] - c["offsets"][:-1]).max()))
    for key, n in (("dx", N), ("dweight", longest), ("dbias", longest)):
        got = getattr(grads, key)
        if got is None:
            continue
        got = got[:P] if key == "dx" else got
        err = (got.double() - want[key]).abs()
        if key == "dbias":
            tol = (n * 2.0 ** -23 + 2.0 ** -16) * size[key] + 2.0 ** -18 * size["slope"]   # the slope's error is not relative: it has a zero
        else:
            tol = 2.0 ** -8 * want[key].abs() + (2.0 ** -8 + n * 2.0 ** -23) * size[key]
        assert (err <= tol + 1e-30).all(), (key, float((err - tol).max()))
    if grads.doperand is not None:
        err = (grads.doperand[:P].double() - want["doperand"]).abs()
        assert (err <= 2.0 ** -8 * want["doperand"].abs() + 2.0 ** -16 * c["dy"][:P].double().abs()).all()
        assert (wdo[0] == 31).all() and (wdo[1 + P:] == 31).all()
    if grads.dx is not None:
        assert (wdx[0] == 31).all() and (wdx[1 + P:] == 31).all()
    assert int(status) == 0
    return grads


@pytest.mark.parametrize("counts", COUNTS, ids=str)
@pytest.mark.parametrize("H,N", [(64, 128), (8, 8), (72, 136), (520, 264), (96, 1024)])
def test_gradients_of_ragged_segments(counts, H, N):
    c = _case(counts, H, N, seed=sum(counts) + N, slack=3)
    _check_backward(c, "silu", "mul")


@pytest.mark.parametrize("name", list(ACTS))
@pytest.mark.parametrize("op", ["none", "add", "mul"])
def test_gradients_through_epilogues(name, op):
    _check_backward(_case([70, 0, 5, 130], 136, 200, slack=9), name, op)


def test_each_gradient_alone_and_the_same_bits_every_time():
    c = _case([90, 0, 200, 33], 264, 520, slack=2)
    whole = _check_backward(c, "gelu", "mul")
    for key in ("dx", "dweight", "dbias", "doperand"):
        alone = _check_backward(c, "gelu", "mul", wanted=(key,))
        a, b = getattr(alone, key), getattr(whole, key)
        assert torch.equal(a[:c["P"]] if key in ("dx", "doperand") else a, b[:c["P"]] if key in ("dx", "doperand") else b), key


def test_gradients_against_differences_of_the_forward_kernel():
    """<dW, D> against the kernel's own forward at W +- h D, both bf16: with values on a coarse grid every product and sum is
    exact, so that the difference is exact as well and only the activation-free product is on trial."""
    counts, H, N = [40, 24], 64, 64
    g = torch.Generator(device="cuda").manual_seed(2)

    def grid(*shape):
        return torch.randint(-2, 3, shape, device="cuda", generator=g).bfloat16()

    off = torch.tensor([0, 40, 64], dtype=torch.int32, device="cuda")
    x, w, dy, d = grid(64, H), grid(2, N, H), grid(64, N), torch.randint(0, 2, (2, N, H), device="cuda", generator=g).bfloat16()
    up, down = (ep.ep_expert_matmul(x, off, w + s * d) for s in (1, -1))
    # |y| <= 64 * 2 * 3 = 384: whole numbers up to 256 are exact in bf16, so keep the columns that stay there
    keep = (up.abs() <= 256) & (down.abs() <= 256)
    dyk = torch.where(keep, dy, torch.zeros_like(dy))
    grads = ep.ep_expert_matmul_backward(dyk, x, off, w)
    _, want = None, float(((up.double() - down.double()) / 2 * dyk.double()).sum())
    exact = plain.experts_gradient(dyk, x, off, w, None)[0]["dweight"]
    assert float((exact * d.double()).sum()) == want
    assert ((grads.dweight.double() - exact).abs() <= 2.0 ** -8 * exact.abs()).all()


def test_operand_may_be_the_output():
    c = _case([50, 200], 128, 192)
    want = ep.ep_expert_matmul(c["x"], c["offsets"], c["weight"], operand=c["operand"], activation=ep.ACT_SILU)
    y = c["operand"].clone()
    ep.ep_expert_matmul(c["x"], c["offsets"], c["weight"], operand=y, activation=ep.ACT_SILU, y=y)
    assert torch.equal(y, want)


def test_offsets_past_the_buffers_are_cut_and_reported():
    c = _case([50, 60], 64, 64)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    x = c["x"][:80].contiguous()
    whole, y = _guarded(80, 64)
    ep.ep_expert_matmul(x, c["offsets"], c["weight"], y=y, status=status)
    assert int(status) == ep.STATUS_CAPACITY and (whole[0] == 31).all() and (whole[-1] == 31).all()
    want = plain.experts(c["x"], c["offsets"], c["weight"])[0][:80]
    assert ((y.double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-3).all()


def test_other_streams_and_graph_replays():
    c = _case([33, 0, 140], 128, 264)
    want = ep.ep_expert_matmul(c["x"], c["offsets"], c["weight"])
    gwant = ep.ep_expert_matmul_backward(c["dy"], c["x"], c["offsets"], c["weight"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = ep.ep_expert_matmul(c["x"], c["offsets"], c["weight"])
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, want)
    y, grads, off = torch.empty_like(want), ep.alloc_expert_grads(c["P"], 128, 264, 3), c["offsets"].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ep.ep_expert_matmul(c["x"], off, c["weight"], y=y)
        ep.ep_expert_matmul_backward(c["dy"], c["x"], off, c["weight"], grads=grads)
    graph.replay()
    assert torch.equal(y, want) and torch.equal(grads.dx, gwant.dx) and torch.equal(grads.dweight, gwant.dweight)
    off.copy_(torch.tensor([0, 100, 101, 173], dtype=torch.int32))              # another routing through the same graph
    graph.replay()
    assert torch.equal(y, ep.ep_expert_matmul(c["x"], off, c["weight"]))
    again = ep.ep_expert_matmul_backward(c["dy"], c["x"], off, c["weight"])
    assert torch.equal(grads.dx, again.dx) and torch.equal(grads.dweight, again.dweight)


def test_rows_past_four_gigabytes():
    """400000 rows of 8192 results: element offsets past 2^31, byte offsets past 2^32, sampled."""
    E, H, N, P = 5, 64, 8192, 400000
    g = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn(P, H, device="cuda", generator=g).bfloat16()
    w = torch.randn(E, N, H, device="cuda", generator=g).bfloat16()
    cut = [0, 90001, 90001, 250000, 399999, 400000]
    off = torch.tensor(cut, dtype=torch.int32, device="cuda")
    y = ep.ep_expert_matmul(x, off, w)
    dx = ep.ep_expert_matmul_backward(y, x, off, w, grads=ep.alloc_expert_grads(P, H, N, E, weight=False)).dx
    for p in (0, 90000, 90001, 249999, 250000, 262143, 262144, 399998, 399999):
        e = max(i for i in range(E) if cut[i] <= p)
        want = w[e].double() @ x[p].double()
        assert ((y[p].double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-4).all(), p
        want, size = y[p].double() @ w[e].double(), y[p].double().abs() @ w[e].double().abs()
        assert ((dx[p].double() - want).abs() <= 2.0 ** -8 * want.abs() + N * 2.0 ** -23 * size).all(), p


@pytest.mark.parametrize("counts,H,N", [([1], 4096, 64), ([5, 0, 40], 2048, 136), ([64, 1], 1032, 264), ([130], 520, 128), ([300, 20], 4104, 72)])
def test_few_tiles_shared_by_several_blocks(counts, H, N):
    """Long contracted axes and few tiles: the axis is cut into up to eight parts, of unequal length and with ragged ends."""
    c = _case(counts, H, N, seed=H, slack=2)
    for name, op in (("none", "none"), ("gelu", "add"), ("silu", "mul")):
        _check_forward(c, name, True, op, pre=True)
    again = [_check_forward(c, "silu", True, "mul") for _ in range(2)]
    assert torch.equal(again[0][:c["P"]], again[1][:c["P"]])


@pytest.mark.parametrize("counts,H,N", [([3000], 64, 72), ([1500, 0, 30], 136, 64), ([900, 1100], 72, 520), ([70, 2500, 1, 0], 128, 128)])
def test_gradients_with_long_segments_and_few_tiles(counts, H, N):
    """The rows are cut into parts; experts without rows, or with fewer rows than parts, among them."""
    _check_backward(_case(counts, H, N, seed=N, slack=5), "silu", "mul")
    _check_backward(_case(counts, N, H * 8, seed=N, slack=5), "gelu", "add")


def test_many_experts():
    """4096 experts, most of them empty."""
    counts = [0] * 4096
    for i, n in ((0, 3), (17, 1), (2000, 90), (4095, 2)):
        counts[i] = n
    c = _case(counts, 64, 72)
    _check_forward(c)
    _check_backward(c, "relu", "none")
