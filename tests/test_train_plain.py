"""The plain statements themselves: the generator's published answers, and the gradients against differences."""
import numpy as np
import torch

import train_plain as plain


def test_philox_gives_its_published_answers():
    """The known answers that the generator's authors publish for ten rounds."""
    for counter, key, want in (
            ((0, 0, 0, 0), (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
            ((0xffffffff,) * 4, (0xffffffff,) * 2, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
            ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0), (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1))):
        got = plain._rounds([np.array([c], np.uint64) for c in counter], *key)
        assert tuple(int(v) for v in got[0]) == want


def test_dropout_keeps_its_share_and_its_mean():
    k = plain.keep(512, 512, 0.3, 77, 5, 1)
    share = float((k > 0).double().mean())
    sigma = (0.3 * 0.7 / 512 ** 2) ** 0.5
    assert abs(share - 0.7) < 5 * sigma and abs(float(k.mean()) - 1.0) < 5 * sigma / 0.7
    for other in (plain.keep(512, 512, 0.3, 78, 5, 1), plain.keep(512, 512, 0.3, 77, 6, 1), plain.keep(512, 512, 0.3, 77, 5, 2)):
        both = float(((k > 0) & (other > 0)).double().mean())        # independent: 0.49
        assert abs(both - 0.49) < 5 * (0.49 * 0.51 / 512 ** 2) ** 0.5
    assert (plain.keep(4, 8, 1.0, 1, 2, 3) == 0).all() and (plain.keep(4, 8, 0.0, 1, 2, 3) == 1).all()


def _difference(f, x, grad, g, eps=1e-6):
    """grad against a central difference of f along a random direction (relative 1e-6: eps^2 and cancellation of 64-bit sums)."""
    d = torch.randn(x.shape, generator=g, dtype=torch.float64)
    num = (f(x + eps * d) - f(x - eps * d)) / (2 * eps)
    assert abs(float(num) - float((grad * d).sum())) <= 1e-6 * max(1.0, abs(float(num)))


def test_row_gradients():
    g = torch.Generator().manual_seed(0)
    T, K, H, P = 5, 3, 16, 11
    slot = torch.tensor([[0, 3, 5], [1, -1, 4], [-1, -1, -1], [2, 2, 6], [10, 9, 8]])      # one row named twice, as by a receive buffer
    x, out, dy = (torch.randn(n, H, generator=g, dtype=torch.float64) for n in (T, P, T))
    d_sorted = torch.randn(P, H, generator=g, dtype=torch.float64)
    w = torch.rand(T, K, generator=g, dtype=torch.float64)
    drop = plain.keep(T, H, 0.25, 9, 1, 0)
    for weights in (w, None):
        _difference(lambda v: (plain.spread(v, slot, weights, P)[0] * d_sorted).sum() if weights is not None else
                    (plain.spread(v, slot, plain.once(slot).double(), P)[0] * d_sorted).sum(), x, plain.gather(d_sorted, slot, weights)[0], g)
    _difference(lambda v: (plain.spread(x, slot, v, P)[0] * d_sorted).sum(), w, plain.dots(x, d_sorted, slot)[0], g)
    _difference(lambda v: (plain.gather(v, slot, w)[0] * drop * dy).sum(), out, plain.spread(dy * drop, slot, w, P)[0], g)
    _difference(lambda v: (plain.gather(out, slot, v)[0] * drop * dy).sum(), w, plain.dots(dy * drop, out, slot)[0], g)


def test_adapter_gradients():
    g = torch.Generator().manual_seed(1)
    n, H, N, r, A = 9, 16, 24, 8, 4
    offsets, index = [0, 3, 3, 7, 8], torch.tensor([4, 0, 7, 1, 2, 8, 3, 5])
    x, base, dy = (torch.randn(n, c, generator=g, dtype=torch.float64) for c in (H, N, N))
    down, up = (torch.randn(A, *s, generator=g, dtype=torch.float64) for s in ((r, H), (N, r)))
    scale = torch.rand(A, generator=g, dtype=torch.float64)

    def f(x, down, up):
        return (plain.adapters(x, base, offsets, index, down, up, scale, 8)[1] * dy).sum()

    mid = plain.adapters(x, base, offsets, index, down, up, scale, 8)[0]
    dx, ddown, dup = plain.adapter_grads(dy, x, torch.zeros(n, H, dtype=torch.float64), offsets, index, down, up, scale, mid)
    _difference(lambda v: f(v, down, up), x, dx, g)
    _difference(lambda v: f(x, v, up), down, ddown, g)
    _difference(lambda v: f(x, down, v), up, dup, g)
