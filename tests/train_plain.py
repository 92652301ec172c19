"""The sort, the combine, dropout and the adapters in 64 bits, with their gradients: plain statements that the kernels are compared with.

Rows are float64 tensors; slots, offsets and indexes int64. Nothing here calls the library."""
import numpy as np
import torch


def philox(seed, step, site, calls):
    """Words of Philox4x32-10 for the counters 0 .. calls - 1: [calls, 4] uint32 (numpy)."""
    low = np.uint64(0xFFFFFFFF)
    v = np.arange(calls, dtype=np.uint64)
    c = [v & low, v >> np.uint64(32), np.full(calls, step & 0xFFFFFFFF, np.uint64), np.full(calls, site, np.uint64)]
    return _rounds(c, seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF)


def _rounds(c, k0, k1):
    low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(10):
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(q >> half) ^ c[1] ^ np.uint64(k0), q & low, (p >> half) ^ c[3] ^ np.uint64(k1), p & low]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return np.stack(c, 1).astype(np.uint32)


def keep(rows, cols, p, seed, step, site):
    """What dropout multiplies the elements of a [rows, cols] array with, in 64 bits; exactly 0 where it drops."""
    edge = int(round(p * 65536))
    w = philox(seed, step, site, rows * cols // 8)
    bits = np.stack([w & 0xFFFF, w >> 16], 2).reshape(rows, cols)
    scale = 0.0 if edge == 65536 else 65536.0 / (65536 - edge)
    return torch.from_numpy(np.where(bits >= edge, scale, 0.0))


def once(slot):
    """Whether a pick is the first of its token that names its row."""
    T, K = slot.shape
    first = torch.ones(T, K, dtype=torch.bool)
    for k in range(1, K):
        first[:, k] = (slot[:, :k] != slot[:, k:k + 1]).all(1)
    return first & (slot >= 0)


def pair_weights(slot, weights):
    """[T, K] factors: the weights; without weights, 1 for the first pick of a row. 0 where the slot is masked."""
    if weights is None:
        return once(slot).double()
    return torch.where(slot >= 0, weights, 0.0)


def spread(v, slot, weights, rows):
    """rows [rows, H]: sum over the picks of a row of w * v[t]; and which rows any pick names."""
    w, out, named = pair_weights(slot, weights), torch.zeros(rows, v.shape[1], dtype=torch.float64), torch.zeros(rows, dtype=torch.bool)
    for k in range(slot.shape[1]):
        t = torch.nonzero(slot[:, k] >= 0).flatten()
        out.index_add_(0, slot[t, k], v[t] * w[t, k, None])
        named[slot[t, k]] = True
    return out, named


def gather(table, slot, weights):
    """[T, H]: sum_k w * table[slot]; and the same of the absolute values."""
    w = pair_weights(slot, weights)
    acc = torch.zeros(slot.shape[0], table.shape[1], dtype=torch.float64)
    mag = torch.zeros_like(acc)
    for k in range(slot.shape[1]):
        t = torch.nonzero(slot[:, k] >= 0).flatten()
        acc[t] += table[slot[t, k]] * w[t, k, None]
        mag[t] += (table[slot[t, k]] * w[t, k, None]).abs()
    return acc, mag


def dots(v, table, slot):
    """[T, K]: <v[t], table[slot]>, 0 where masked; and the same of the absolute values."""
    out = torch.zeros(slot.shape, dtype=torch.float64)
    mag = torch.zeros_like(out)
    for k in range(slot.shape[1]):
        t = torch.nonzero(slot[:, k] >= 0).flatten()
        out[t, k] = (v[t] * table[slot[t, k]]).sum(1)
        mag[t, k] = (v[t] * table[slot[t, k]]).abs().sum(1)
    return out, mag


def entries(offsets, index):
    """[(adapter, entry numbers, rows)] of the adapters that have some."""
    found = []
    for a in range(len(offsets) - 1):
        e = torch.arange(int(offsets[a]), int(offsets[a + 1]))
        if len(e):
            found.append((a, e, e if index is None else index[e]))
    return found


def adapters(x, base, offsets, index, down, up, scale, count):
    """mid [count, r] (0 where no entry is) and y."""
    mid, y = torch.zeros(count, down.shape[1], dtype=torch.float64), base.clone()
    for a, e, row in entries(offsets, index):
        mid[e] = x[row] @ down[a].t()
        y[row] = base[row] + scale[a] * (mid[e] @ up[a].t())
    return mid, y


def adapter_grads(dy, x, base, offsets, index, down, up, scale, mid):
    """dx, ddown, dup for dy, from a given mid."""
    dx, ddown, dup = base.clone(), torch.zeros_like(down), torch.zeros_like(up)
    for a, e, row in entries(offsets, index):
        dmid = scale[a] * (dy[row] @ up[a])
        dx[row] = base[row] + dmid @ down[a]
        ddown[a] = dmid.t() @ x[row]
        dup[a] = scale[a] * (dy[row].t() @ mid[e])
    return dx, ddown, dup
