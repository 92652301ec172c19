"""The forms of the experts' products that batches of real size take, compared in full: pairs of CTAs with several tiles each, whose
second CTA holds real features, whose ring of stages wraps, and with every epilogue; single CTAs with several tiles each. The
tolerances are those of `test_gpu_experts`."""
import pytest
import torch

from test_gpu_experts import ACTS, _case, _check_backward, _check_forward

pytestmark = pytest.mark.gpu


def _ragged(E, low, high, seed, **fixed):
    c = torch.randint(low, high + 1, (E,), generator=torch.Generator().manual_seed(seed)).tolist()
    for e, n in fixed.items():
        c[int(e[1:])] = n
    return c


# some 250 rows per expert: 256 columns a tile; one segment longer than the ring's stages, some of a few rows, two without any
PAIRS = _ragged(40, 100, 400, 1, e3=0, e4=1, e17=700, e25=17, e38=257, e39=0)
# some 100 rows per expert: 128 columns a tile
NARROW = _ragged(33, 60, 120, 2, e0=0, e7=129, e32=1)
# some 25 rows per expert: 64 columns, single CTAs
FEW = _ragged(44, 0, 40, 3, e1=65, e43=130)


def _takes_pairs(counts, M):
    E, P = len(counts), sum(counts)
    columns = 64
    while columns < 256 and columns * E < P + P // 2:
        columns *= 2
    return columns >= 128 and (min(P, E) + P // columns) * -(-M // 256) >= 74


def test_cases_are_of_the_form_they_are_meant_for():
    for counts in (PAIRS, NARROW):
        for M in (520, 1032, 1160):
            assert _takes_pairs(counts, M)
    assert not _takes_pairs(FEW, 1160)
    tiles = sum(-(-n // 64) for n in FEW)
    assert tiles * -(-520 // 128) > 148 and tiles * -(-1160 // 128) > 300


@pytest.mark.parametrize("counts", [PAIRS, NARROW, FEW], ids=["pairs", "narrow", "few"])
@pytest.mark.parametrize("name", list(ACTS))
@pytest.mark.parametrize("op", ["none", "add", "mul"])
@pytest.mark.parametrize("bias,pre", [(False, False), (True, False), (True, True)])
def test_epilogues_of_many_tiles(counts, name, op, bias, pre):
    _check_forward(_case(counts, 520, 1032, seed=7, slack=9), name, bias, op, pre=pre)


@pytest.mark.parametrize("counts", [PAIRS, NARROW, FEW], ids=["pairs", "narrow", "few"])
@pytest.mark.parametrize("H,N", [(1160, 520), (72, 2056), (264, 1536)])
def test_products_of_many_tiles(counts, H, N):
    _check_forward(_case(counts, H, N, seed=8, slack=3), "silu", True, "mul", pre=True)


@pytest.mark.parametrize("counts", [PAIRS, NARROW, FEW], ids=["pairs", "narrow", "few"])
@pytest.mark.parametrize("H,N", [(520, 1032), (1160, 520), (1536, 264)])
@pytest.mark.parametrize("name,op", [("none", "none"), ("silu", "mul"), ("gelu", "add"), ("relu", "mul")])
def test_gradients_of_many_tiles(counts, H, N, name, op):
    _check_backward(_case(counts, H, N, seed=9, slack=9), name, op)


@pytest.mark.parametrize("name,op", [("none", "none"), ("silu", "mul")])
def test_weight_gradients_of_single_blocks(name, op):
    """Six experts of 520 x 520: 150 tiles of 128 columns, one CTA each."""
    _check_backward(_case([200, 0, 450, 64, 65, 131], 520, 520, seed=10, slack=5), name, op)
