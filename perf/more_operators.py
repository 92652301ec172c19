"""Rows sorted by expert and back with their gradients, dropout, and low-rank adapters: what they are measured on.

Each case is one pass through one operator. With `own` false, `run` computes it in plain torch operations in 32 bits,
rounded once at the end; with `own` true it makes the calls a user makes of `paper_2609_40093_b200.ep`.

    sort      sorted[slot[t][k]] = w[t][k] * x[t] in the pair space; with grad also, for d_sorted, dx[t] = add[t] + sum_k w[t][k] *
              d_sorted[slot[t][k]] and d_weights[t][k] = <x[t], d_sorted[slot[t][k]]>
    combine   y[t] = residual[t] + drop(sum_k w[t][k] * out[slot[t][k]]); with grad also, for dy, d_out[slot[t][k]] = w[t][k] * drop(dy[t])
              and d_weights[t][k] = <drop(dy[t]), out[slot[t][k]]>
    dropout   y = residual + drop(x) over the first `limit` rows; with grad also the gradient of x, drop(dy)
    adapters  y[row] = base[row] + scale[a] * (x[row] down[a]^T) up[a]^T for the rows of adapter a
    adapter_grads   its gradients: dx (added to what the shared projection gives), ddown and dup

drop(v) keeps an element where its 16 bits of Philox4x32-10 (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2,
3", 2011) reach round(65536 p), and scales what it keeps by 1 / (1 - round(65536 p) / 65536). The eight elements 8 v .. 8 v + 7 of a row-major
array share one call: counter (low word of v, high word of v, step, site), key (low and high word of the seed); the elements
take the low and the high half of the first word, of the second, and so on.
"""
import math

import numpy as np
import torch

own = False


# ---------------------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # a decode batch of 64 tokens, 2 of 8 experts, weights applied before the experts: latency
        dict(name="sort_decode", op="sort", T=64, K=2, E=8, H=4096, masked=0.0, weighted=True, add=False, grad=False),
        # a training step of 4096 tokens, 8 of 128 experts: the two branches of a gated expert give two gradients, one is added to the other
        dict(name="sort_train", op="sort", T=4096, K=8, E=128, H=2048, masked=0.02, weighted=True, add=True, grad=True),
        # a ragged training batch with padding tokens, a width that is no multiple of a cache line
        dict(name="combine_ragged", op="combine", T=1003, K=6, E=60, H=520, masked=0.05, residual=True, p=0.0, grad=True),
        # the largest layer: 8192 tokens of 7168 elements, 8 of 256 experts, residual and dropout
        dict(name="combine_large", op="combine", T=8192, K=8, E=256, H=7168, masked=0.0, residual=True, p=0.1, grad=True),
        # the hidden rows of a small batch
        dict(name="dropout_small", op="dropout", rows=1003, cols=264, limit=0.9, residual=False, p=0.4, grad=True),
        # the hidden rows of 4096 tokens with 8 picks
        dict(name="dropout_hidden", op="dropout", rows=32768, cols=1024, limit=0.98, residual=False, p=0.1, grad=True),
        # residual and dropout of 65536 tokens
        dict(name="dropout_large", op="dropout", rows=65536, cols=7168, limit=1.0, residual=True, p=0.1, grad=False),
        # one token being generated with one of 32 adapters resident
        dict(name="adapters_one_token", op="adapters", rows=1, H=4096, N=4096, A=32, r=16, order="mixed", without=0.0, mid=False),
        # a decode batch of 256 requests in any order, 64 adapters, a tenth of the requests without one
        dict(name="adapters_decode", op="adapters", rows=256, H=2048, N=8192, A=64, r=16, order="mixed", without=0.1, mid=False),
        # a training batch of 16384 tokens, four adapters, each its own block of tokens
        dict(name="adapters_train", op="adapters", rows=16384, H=4096, N=8192, A=4, r=64, order="segments", without=0.0, mid=True),
        # a small fine-tuning step, odd sizes, adapters without rows
        dict(name="adapter_grads_ragged", op="adapter_grads", rows=1003, H=520, N=264, A=12, r=24, order="mixed", without=0.1),
        # every expert its adapter: the pair space of 4096 tokens, 8 of 128 experts
        dict(name="adapter_grads_experts", op="adapter_grads", rows=32768, H=2048, N=1024, A=128, r=32, order="segments", without=0.0),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("sort", "combine", "dropout", "adapters", "adapter_grads"))
    if op in ("sort", "combine"):
        while True:
            T, K, H = _log_int(rng, 1, 16384), rng.randint(1, 12), 8 * _log_int(rng, 4, 896)
            if T * K * H <= 4.6e8:
                break
        c = dict(op=op, T=T, K=K, E=rng.randint(K, 256), H=H, masked=rng.choice((0.0, 0.05)), grad=rng.random() < 0.7)
        if op == "sort":
            return dict(c, weighted=rng.random() < 0.6, add=rng.random() < 0.5)
        return dict(c, residual=rng.random() < 0.6, p=rng.choice((0.0, 0.1, 0.37)))
    if op == "dropout":
        while True:
            rows, cols = _log_int(rng, 1, 65536), 8 * _log_int(rng, 4, 1024)
            if rows * cols <= 2.3e8:
                break
        return dict(op=op, rows=rows, cols=cols, limit=rng.choice((1.0, 0.7)), residual=rng.random() < 0.5, p=rng.choice((0.05, 0.1, 0.5)), grad=rng.random() < 0.5)
    while True:
        rows, H, N = _log_int(rng, 1, 32768), 8 * _log_int(rng, 8, 896), 8 * _log_int(rng, 8, 1024)
        A, r = _log_int(rng, 1, 256), 8 * _log_int(rng, 1, 16)
        if rows * (H + 2 * N) <= (3.3e8 if op == "adapters" else 1.3e8) and A * r * (H + N) <= 2e8:
            break
    c = dict(op=op, rows=rows, H=H, N=N, A=A, r=r, order=rng.choice(("mixed", "segments")), without=rng.choice((0.0, 0.2)))
    return dict(c, mid=rng.random() < 0.5) if op == "adapters" else c


def _adapter_rows(case, seed):
    """Rows of each adapter: A whole numbers whose sum is at most `rows`; the others have none."""
    r = np.random.RandomState(seed % (1 << 32))
    p = (r.permutation(case["A"]) + 1.0) ** -0.7                     # some adapters are asked for more often
    return r.multinomial(case["rows"] - int(case["rows"] * case["without"]), p / p.sum())


# --------------------------------------------------------------------------------------------------------- inputs

def prepare(case, seed):
    dev, bf = torch.device("cuda"), torch.bfloat16
    g = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape, dtype=bf, scale=1.0):
        t = torch.empty(*shape, dtype=dtype, device=dev)
        t.normal_(0.0, scale, generator=g)
        return t

    c = dict(case)
    s = {"case": c}
    if c["op"] in ("sort", "combine"):
        T, K, E, H = c["T"], c["K"], c["E"], c["H"]
        liked = normal(E, dtype=torch.float32, scale=0.7)
        idx = torch.topk(normal(T, E, dtype=torch.float32) + liked, K, dim=1).indices
        weights = torch.softmax(normal(T, K, dtype=torch.float32), 1)
        if c["masked"]:                                              # padding tokens, and single picks that were dropped
            dead = torch.rand(T, 1, generator=g, device=dev) < c["masked"]
            dead = dead | (torch.rand(T, K, generator=g, device=dev) < 0.1 * c["masked"])
            idx = torch.where(dead, -1, idx)
        key = torch.where(idx < 0, E, idx).flatten()                 # pairs by expert, in the order of (token, pick) within one
        order = torch.argsort(key, stable=True)
        slot = torch.empty(T * K, dtype=torch.int32, device=dev)
        slot[order] = torch.arange(T * K, dtype=torch.int32, device=dev)
        s["slot"] = torch.where(idx.flatten() < 0, -1, slot).view(T, K)
        s["weights"] = weights if c.get("weighted", True) else None
        if c["op"] == "sort":
            s["x"] = normal(T, H)
            if c["grad"]:
                s["d_sorted"] = normal(T * K, H)
                s["add"] = normal(T, H) if c["add"] else None
        else:
            s["out"] = normal(T * K, H)
            s["residual"] = normal(T, H) if c["residual"] else None
            if c["grad"]:
                s["dy"] = normal(T, H)
    elif c["op"] == "dropout":
        s["x"] = normal(c["rows"], c["cols"])
        s["residual"] = normal(c["rows"], c["cols"]) if c["residual"] else None
        s["live"] = max(1, int(c["rows"] * c["limit"]))
        s["limit"] = torch.tensor([s["live"]], dtype=torch.int32, device=dev) if c["limit"] < 1.0 else None
        if c["grad"]:
            s["dy"] = normal(c["rows"], c["cols"])
    else:
        n, H, N, A, r = c["rows"], c["H"], c["N"], c["A"], c["r"]
        off = np.concatenate([[0], np.cumsum(_adapter_rows(c, seed))])
        s["segments"] = [int(v) for v in off]
        s["offsets"] = torch.from_numpy(off.astype(np.int32)).to(dev)
        # mixed: the batch's rows in any order; entry i of the sorted list is row index[i], what is behind the last one names no row
        s["index"] = None
        if c["order"] == "mixed":
            s["index"] = torch.randperm(n, generator=g, device=dev).to(torch.int32)
        s["x"] = normal(n, H)
        s["down"] = normal(A, r, H, scale=H ** -0.5)
        s["up"] = normal(A, N, r, scale=r ** -0.5)
        s["scale"] = 0.5 + torch.rand(A, generator=g, device=dev)
        if c["op"] == "adapters":
            s["base"] = normal(n, N)
        else:
            s["dy"] = normal(n, N)
            s["mid"] = normal(n, r)
            s["base"] = normal(n, H)
    if c.get("p"):
        s["random"] = torch.tensor([(seed * 0x9E3779B97F4A7C15 + 12345) % (1 << 63), 1 + seed % 1000], dtype=torch.int64, device=dev)    # seed and step
        s["site"] = 3
    return s


# ----------------------------------------------------------------------------------------------------- plain forms

_LOW = 0xFFFFFFFF


def _philox(state, site, calls, device):
    """The four words of Philox4x32-10 for the counters 0 .. calls - 1, [calls, 4] in int64 (whose products wrap, their bits are right)."""
    v = torch.arange(calls, dtype=torch.int64, device=device)
    c0, c1, c2, c3 = v & _LOW, v >> 32, (state[1] & _LOW).expand(calls), torch.full((calls,), site, dtype=torch.int64, device=device)
    k0, k1 = state[0] & _LOW, (state[0] >> 32) & _LOW
    for i in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & _LOW) ^ c1 ^ ((k0 + i * 0x9E3779B9) & _LOW), b & _LOW, ((a >> 32) & _LOW) ^ c3 ^ ((k1 + i * 0xBB67AE85) & _LOW), a & _LOW
    return torch.stack([c0, c1, c2, c3], 1)


def _plain_drop(s, v):
    """v (float32) with its dropped elements at 0 and the others scaled."""
    p = s["case"]["p"]
    if not p:
        return v
    edge = int(round(p * 65536))
    w = _philox(s["random"], s["site"], v.numel() // 8, v.device)
    kept = torch.stack([(w & 0xFFFF) >= edge, (w >> 16) >= edge], 2).view(v.shape)
    return torch.where(kept, v * (65536.0 / (65536 - edge)), 0.0)


def _rows_of(table, slot):
    """table[slot[t][k]] in 32 bits, [T, K, H], zeros where the slot is -1."""
    return torch.where((slot >= 0).unsqueeze(2), table[slot.clamp(min=0).long()].float(), 0.0)


def _to_pairs(rows, slot, like):
    """rows [T, K, H] to their places in a table of zeros."""
    out = torch.zeros_like(like)
    there = (slot >= 0).flatten()
    out[slot.flatten()[there].long()] = rows.to(out.dtype).flatten(0, 1)[there]
    return out


def _plain_sort(s):
    c, slot, x = s["case"], s["slot"], s["x"].float()
    w = (torch.ones_like(slot, dtype=torch.float32) if s["weights"] is None else s["weights"]).unsqueeze(2)
    like = torch.empty(c["T"] * c["K"], c["H"], dtype=torch.bfloat16, device=x.device)
    out = {"sorted": _to_pairs(x.unsqueeze(1) * w, slot, like)}
    if c["grad"]:
        g = _rows_of(s["d_sorted"], slot)
        dx = (g * w).sum(1)
        out["dx"] = (dx if s["add"] is None else dx + s["add"].float()).to(torch.bfloat16)
        if s["weights"] is not None:
            out["d_weights"] = (g * x.unsqueeze(1)).sum(2)
    return out


def _plain_combine(s):
    c, slot, w = s["case"], s["slot"], s["weights"].unsqueeze(2)
    rows = _rows_of(s["out"], slot)
    y = _plain_drop(s, (rows * w).sum(1))
    out = {"y": (y if s["residual"] is None else y + s["residual"].float()).to(torch.bfloat16)}
    if c["grad"]:
        g = _plain_drop(s, s["dy"].float()).unsqueeze(1)
        out["d_weights"] = (rows * g).sum(2)
        out["d_out"] = _to_pairs(g * w, slot, s["out"])
    return out


def _plain_dropout(s):
    c, n = s["case"], s["live"]

    def one(v, residual):
        d = _plain_drop(s, v[:n].float())
        y = torch.zeros_like(v)
        y[:n] = d if residual is None else d + residual[:n].float()
        return y

    out = {"y": one(s["x"], s["residual"])}
    if c["grad"]:
        out["dx"] = one(s["dy"], None)
    return out


def _entries(s):
    """(rows in the order of their adapters, the adapter of each) as index tensors."""
    n, dev = s["segments"][-1], s["x"].device
    rows = torch.arange(n, device=dev) if s["index"] is None else s["index"][:n].long()
    count = (s["offsets"][1:] - s["offsets"][:-1]).long()
    return rows, torch.repeat_interleave(torch.arange(s["case"]["A"], device=dev), count, output_size=n)


def _plain_adapters(s):
    c = s["case"]
    rows, which = _entries(s)
    y, mid = s["base"].clone(), torch.zeros(c["rows"], c["r"], dtype=torch.bfloat16, device=rows.device)
    if len(rows) * c["r"] * (c["H"] + c["N"]) <= 1 << 28:             # few rows: every row its own weights, one batched product
        m = torch.bmm(s["down"][which].float(), s["x"][rows].float().unsqueeze(2))
        mid[:len(rows)] = m.squeeze(2)
        d = torch.bmm(s["up"][which].float(), m).squeeze(2) * s["scale"][which].unsqueeze(1)
        y[rows] = (d + s["base"][rows].float()).to(torch.bfloat16)
    else:                                                            # one product an adapter: the segments differ in length
        for a in range(c["A"]):
            i, j = s["segments"][a], s["segments"][a + 1]
            if i < j:
                m = s["x"][rows[i:j]].float() @ s["down"][a].float().t()
                mid[i:j] = m
                y[rows[i:j]] = (s["base"][rows[i:j]].float() + s["scale"][a] * (m @ s["up"][a].float().t())).to(torch.bfloat16)
    return {"y": y, "mid": mid} if c["mid"] else {"y": y}


def _plain_adapter_grads(s):
    c = s["case"]
    rows, _ = _entries(s)
    out = {"dx": s["base"].clone(), "ddown": torch.zeros_like(s["down"]), "dup": torch.zeros_like(s["up"])}
    for a in range(c["A"]):
        i, j = s["segments"][a], s["segments"][a + 1]
        if i < j:
            g, x, m = s["dy"][rows[i:j]].float() * s["scale"][a], s["x"][rows[i:j]].float(), s["mid"][i:j].float()
            dm = g @ s["up"][a].float()
            out["dx"][rows[i:j]] = (s["base"][rows[i:j]].float() + dm @ s["down"][a].float()).to(torch.bfloat16)
            out["ddown"][a] = dm.t() @ x
            out["dup"][a] = g.t() @ m
    return out


# ------------------------------------------------------------------------------------------------------------ run

def _own_buffers(s):
    """What a program allocates once for a shape and keeps: outputs and workspaces."""
    from paper_2609_40093_b200 import ep
    c, bf = s["case"], torch.bfloat16
    s["drop"] = ep.Dropout(c["p"], s["random"], site=s["site"]) if c.get("p") else None
    if c["op"] == "sort":
        s["sorted"] = torch.zeros(c["T"] * c["K"], c["H"], dtype=bf, device="cuda")
        if c["grad"]:
            s["dx"] = torch.empty_like(s["x"])
            s["d_weights"] = torch.empty_like(s["weights"]) if s["weights"] is not None else None
    elif c["op"] == "combine":
        s["y"] = torch.empty(c["T"], c["H"], dtype=bf, device="cuda")
        if c["grad"]:
            s["d_out"], s["d_weights"] = torch.zeros_like(s["out"]), torch.empty_like(s["weights"])
    elif c["op"] == "dropout":
        s["y"] = torch.zeros_like(s["x"])
        s["dx"] = torch.zeros_like(s["x"]) if c["grad"] else None
    else:
        s["adapters"] = ep.Adapters(s["down"], s["up"], s["scale"])
        if c["op"] == "adapters":
            s["y"] = s["base"].clone()                               # rows without an adapter are not touched
            s["mid"] = torch.zeros(c["rows"], c["r"], dtype=bf, device="cuda") if c["mid"] else None
        else:
            s["grads"] = ep.alloc_adapter_grads(s["x"], s["adapters"], entries=c["rows"])
            s["grads"].dx.copy_(s["base"])
    s["ready"] = True


def _own_run(s):
    from paper_2609_40093_b200 import ep
    c = s["case"]
    if "ready" not in s:
        _own_buffers(s)
    if c["op"] == "sort":
        out = {"sorted": ep.ep_sort(s["x"], s["slot"], s["sorted"], weights=s["weights"])}
        if c["grad"]:
            weighted = s["weights"] is not None
            out["dx"] = ep.ep_sort_backward(s["d_sorted"], s["slot"], s["dx"], weights=s["weights"], x=s["x"] if weighted else None,
                                            d_weights=s["d_weights"], add=s["add"])
            if weighted:
                out["d_weights"] = s["d_weights"]
        return out
    if c["op"] == "combine":
        out = {"y": ep.ep_combine_residual(s["out"], s["slot"], s["weights"], s["y"], residual=s["residual"], dropout=s["drop"])}
        if c["grad"]:
            out["d_out"] = ep.ep_combine_backward(s["dy"], s["slot"], s["weights"], s["d_out"], out=s["out"], d_weights=s["d_weights"], dropout=s["drop"])
            out["d_weights"] = s["d_weights"]
        return out
    if c["op"] == "dropout":
        out = {"y": ep.ep_dropout(s["x"], s["drop"], residual=s["residual"], y=s["y"], limit=s["limit"])}
        if c["grad"]:
            out["dx"] = ep.ep_dropout(s["dy"], s["drop"], y=s["dx"], limit=s["limit"])
        return out
    if c["op"] == "adapters":
        y = ep.ep_adapter_matmul(s["x"], s["offsets"], s["adapters"], s["y"], base=s["base"], row_index=s["index"], mid=s["mid"])
        return {"y": y, "mid": s["mid"]} if c["mid"] else {"y": y}
    g = ep.ep_adapter_matmul_backward(s["dy"], s["x"], s["offsets"], s["adapters"], s["mid"], s["grads"], base=s["base"], row_index=s["index"])
    return {"dx": g.dx, "ddown": g.ddown, "dup": g.dup}


def run(state):
    if own:
        return _own_run(state)
    return {"sort": _plain_sort, "combine": _plain_combine, "dropout": _plain_dropout, "adapters": _plain_adapters,
            "adapter_grads": _plain_adapter_grads}[state["case"]["op"]](state)


# ----------------------------------------------------------------------------------------------------------- work

def work(case):
    c = case
    if c["op"] in ("sort", "combine"):
        T, K, H = c["T"], c["K"], c["H"]
        P = int(T * K * (1 - c["masked"]))
        if c["op"] == "sort":
            w = 4 * T * K if c["weighted"] else 0
            bytes_, flops = 2 * (T + P) * H + 4 * T * K + w, P * H
            if c["grad"]:                                            # a pass of its own, later in a step
                bytes_ += 2 * (P + T + (T if c["add"] else 0) + (T if c["weighted"] else 0)) * H + 4 * T * K + 2 * w
                flops += 4 * P * H
            return {"bytes": bytes_, "flops": flops}
        bytes_, flops = 2 * (P + T + (T if c["residual"] else 0)) * H + 8 * T * K, 2 * P * H
        if c["grad"]:
            bytes_, flops = bytes_ + 2 * (2 * P + T) * H + 12 * T * K, flops + 3 * P * H
        return {"bytes": bytes_, "flops": flops}
    if c["op"] == "dropout":
        n = max(1, int(c["rows"] * c["limit"])) * c["cols"]
        return {"bytes": 2 * n * (2 + (1 if c["residual"] else 0) + (2 if c["grad"] else 0)), "flops": n * (2 if c["grad"] else 1)}
    counts = _adapter_rows(c, 0)
    n, live, H, N, r = int(counts.sum()), int((counts > 0).sum()), c["H"], c["N"], c["r"]
    index = 4 * (c["A"] + 1) + (4 * n if c["order"] == "mixed" else 0)
    if c["op"] == "adapters":
        return {"bytes": 2 * n * (H + 2 * N) + 2 * live * r * (H + N) + (2 * n * r if c["mid"] else 0) + 4 * c["A"] + index, "flops": 2 * n * r * (H + N)}
    return {"bytes": 2 * n * (N + 3 * H + r) + 2 * (live + c["A"]) * r * (H + N) + 4 * c["A"] + index, "flops": 4 * n * r * (H + N)}


# ---------------------------------------------------------------------------------------------------- in 64 bits

def _exact_keep(s, shape):
    """What drop() multiplies with, in 64 bits: the generator once more, its products made of 16-bit halves."""
    n, dev = math.prod(shape) // 8, s["slot"].device if "slot" in s else s["x"].device
    word = torch.arange(n, device=dev)
    seed, step = (int(v) for v in s["random"].tolist())
    ctr = [word % 2 ** 32, torch.div(word, 2 ** 32, rounding_mode="floor"), torch.full_like(word, step % 2 ** 32), torch.full_like(word, s["site"])]
    key = [seed % 2 ** 32, (seed >> 32) % 2 ** 32]

    def product(m, v):
        """High and low word of the product of two unsigned words."""
        low, high = (v % 65536) * m, torch.div(v, 65536, rounding_mode="floor") * m
        mid = torch.div(low, 65536, rounding_mode="floor") + high
        return torch.div(mid, 65536, rounding_mode="floor"), (mid % 65536) * 65536 + low % 65536

    for _ in range(10):
        (ha, la), (hb, lb) = product(0xD2511F53, ctr[0]), product(0xCD9E8D57, ctr[2])
        ctr = [hb ^ ctr[1] ^ key[0], lb, ha ^ ctr[3] ^ key[1], la]
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    edge = int(round(s["case"]["p"] * 65536))
    keep = torch.empty(n, 8, dtype=torch.float64, device=dev)
    for i in range(4):
        keep[:, 2 * i] = (ctr[i] % 65536 >= edge).double()
        keep[:, 2 * i + 1] = (torch.div(ctr[i], 65536, rounding_mode="floor") >= edge).double()
    return keep.view(shape) / (1.0 - edge / 65536)


def exact(case, seed):
    s, c, d64 = prepare(case, seed), case, dict(dtype=torch.float64, device="cuda")
    if c["op"] in ("sort", "combine"):
        T, K, H = c["T"], c["K"], c["H"]
        w = torch.ones(T, K, **d64) if s["weights"] is None else s["weights"].double()
        token, pick = torch.nonzero(s["slot"] >= 0, as_tuple=True)
        place = s["slot"][token, pick].long()
        keep = _exact_keep(s, (T, H)) if c.get("p") else torch.ones(1, 1, **d64)
        acc, dots, spread = torch.zeros(T, H, **d64), torch.zeros(T, K, **d64), torch.zeros(T * K, H, **d64)
        table = s["d_sorted"] if c["op"] == "sort" and c["grad"] else s.get("out")
        rows = s["x"] if c["op"] == "sort" else s.get("dy")
        for k in range(K):                                           # a pick at a time keeps the 64-bit rows small
            m = pick == k
            t, q = token[m], place[m]
            if rows is not None:
                v = rows[t].double()
                if c["op"] == "combine" and c.get("p"):
                    v = v * keep[t]
                spread[q] = v * w[t, k, None]
            if table is not None:
                u = table[q].double()
                acc[t] += u * w[t, k, None]
                if rows is not None:
                    dots[t, k] = (u * v).sum(1)
        if c["op"] == "sort":
            out = {"sorted": spread}
            if c["grad"]:
                out["dx"] = acc if s["add"] is None else acc + s["add"].double()
                if s["weights"] is not None:
                    out["d_weights"] = dots
            return out
        y = acc * keep
        out = {"y": y if s["residual"] is None else y + s["residual"].double()}
        if c["grad"]:
            out["d_out"], out["d_weights"] = spread, dots
        return out
    if c["op"] == "dropout":
        keep, n = _exact_keep(s, (s["live"], c["cols"])), s["live"]
        y = torch.zeros(c["rows"], c["cols"], **d64)
        y[:n] = s["x"][:n].double() * keep
        if s["residual"] is not None:
            y[:n] += s["residual"][:n].double()
        if not c["grad"]:
            return {"y": y}
        dx = torch.zeros(c["rows"], c["cols"], **d64)
        dx[:n] = s["dy"][:n].double() * keep
        return {"y": y, "dx": dx}
    rows = [list(range(*s["segments"][a:a + 2])) for a in range(c["A"])]
    place = torch.arange(c["rows"]) if s["index"] is None else s["index"].long().cpu()
    result = s["base"].double()
    if c["op"] == "adapters":
        mid = torch.zeros(c["rows"], c["r"], **d64)
        for a, e in enumerate(rows):
            if e:
                p = place[e[0]:e[-1] + 1].cuda()
                mid[e[0]:e[-1] + 1] = torch.mm(s["x"][p].double(), s["down"][a].double().t())
                result[p] += s["scale"][a].double() * torch.mm(mid[e[0]:e[-1] + 1], s["up"][a].double().t())
        return {"y": result, "mid": mid} if c["mid"] else {"y": result}
    ddown, dup = torch.zeros(c["A"], c["r"], c["H"], **d64), torch.zeros(c["A"], c["N"], c["r"], **d64)
    for a, e in enumerate(rows):
        if e:
            p = place[e[0]:e[-1] + 1].cuda()
            g = s["dy"][p].double() * s["scale"][a].double()
            inner = torch.mm(g, s["up"][a].double())
            result[p] += torch.mm(inner, s["down"][a].double())
            ddown[a] = torch.mm(inner.t(), s["x"][p].double())
            dup[a] = torch.mm(g.t(), s["mid"][e[0]:e[-1] + 1].double())
    return {"dx": result, "ddown": ddown, "dup": dup}
