"""The router, the balance loss and the experts' matrix products: what they are measured on.

Each case is one pass through one operator. With `own` false, `run` computes it in plain torch operations in 32 bits,
rounded once at the end; with `own` true it makes the calls a user makes of `paper_2609_40093_b200.ep`.

    route     logits [T, E] -> topk_idx [T, K] (descending score, ties to the lowest id, -1 where no expert is left)
              and topk_weights [T, K], the tables that layout, dispatch and combine take
    train     the same plus expert counts, mean probabilities and balance loss, then the gradient of both the weights
              and the loss with respect to the logits
    experts   y[p] = act(x[p] W[e]^T + b[e]) (+ or *) operand[p] for the rows p of expert e in the pair space
    backward  its gradients: dx, dweight, dbias and, where the operand multiplies, doperand
"""
import math

import numpy as np
import torch

own = False

ACTS = ("none", "relu", "silu", "gelu")


# ---------------------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # a decode batch of 64 tokens on 8 experts: pure latency
        dict(name="route_decode", op="route", T=64, E=8, K=2, dtype="f32", scoring="softmax", renorm=True, bias=False, scale=1.0, masked=0.0),
        # a prefill batch of 8 of 128 experts on 16-bit logits: equal logits are common, ties decide
        dict(name="route_prefill_bf16", op="route", T=4096, E=128, K=8, dtype="bf16", scoring="softmax", renorm=True, bias=False, scale=1.0, masked=0.02),
        # 8 of 256 experts, sigmoid scores with a per-expert selection bias and scaled weights
        dict(name="route_sigmoid_bias", op="route", T=8192, E=256, K=8, dtype="f32", scoring="sigmoid", renorm=True, bias=True, scale=2.5, masked=0.0),
        # a ragged training batch, an expert count that is no multiple of a vector, weights not renormalised, padding rows
        dict(name="train_ragged", op="train", T=1003, E=60, K=6, dtype="bf16", scoring="softmax", renorm=False, bias=False, scale=1.0, masked=0.05),
        # a training batch of 8 of 128 experts
        dict(name="train_mid", op="train", T=4096, E=128, K=8, dtype="f32", scoring="softmax", renorm=True, bias=False, scale=1.0, masked=0.0),
        # the largest routing table: 65536 tokens on 256 experts, sigmoid scores
        dict(name="train_large", op="train", T=65536, E=256, K=8, dtype="f32", scoring="sigmoid", renorm=True, bias=True, scale=2.5, masked=0.01),
        # one token being generated: two experts of one row each, the time of reading their weights
        dict(name="experts_one_token", op="experts", P=2, H=4096, N=8192, E=8, skew="spread", act="silu", bias=False, operand="mul"),
        # a decode batch of 256 tokens, 8 of 128 experts: some sixteen rows an expert
        dict(name="experts_decode", op="experts", P=2048, H=2048, N=1024, E=128, skew="uniform", act="silu", bias=True, operand="none"),
        # a prefill batch of 8192 tokens, 8 of 256 experts, one hot expert: bound by the tensor cores
        dict(name="experts_prefill", op="experts", P=65536, H=7168, N=2048, E=256, skew="burst", act="silu", bias=False, operand="mul"),
        # a small training step with odd sizes, experts without rows, an added operand
        dict(name="backward_ragged", op="backward", P=1003, H=520, N=264, E=12, skew="zipf", act="gelu", bias=True, operand="add"),
        # a training step of 4096 tokens, 8 of 128 experts, skewed
        dict(name="backward_mid", op="backward", P=32768, H=2048, N=1024, E=128, skew="zipf", act="silu", bias=True, operand="mul"),
        # long segments: 8 experts of some 2048 rows each
        dict(name="backward_large", op="backward", P=16384, H=4096, N=8192, E=8, skew="uniform", act="silu", bias=False, operand="mul"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("route", "train", "experts", "backward"))
    if op in ("route", "train"):
        E = _log_int(rng, 4, 1024)
        T = _log_int(rng, 1, min(65536, (1 << 24) // E))
        scoring = rng.choice(("softmax", "sigmoid"))
        return dict(op=op, T=T, E=E, K=rng.randint(1, min(E, 12)), dtype=rng.choice(("f32", "bf16")), scoring=scoring, renorm=rng.random() < 0.6,
                    # with softmax scores a selection bias makes the order hang on the last bits of a sum over the experts
                    bias=scoring == "sigmoid" and rng.random() < 0.5, scale=rng.choice((1.0, 2.5)), masked=rng.choice((0.0, 0.03)))
    while True:
        E, P = _log_int(rng, 1, 256), _log_int(rng, 1, 65536)
        H, N = 8 * _log_int(rng, 8, 896), 8 * _log_int(rng, 8, 1024)
        if P * H * N <= (9.6e11 if op == "experts" else 5.4e11) and E * H * N <= (3.7e9 if op == "experts" else 2.6e8) and P * max(H, N) <= 4.8e8:
            return dict(op=op, P=P, H=H, N=N, E=E, skew=rng.choice(("uniform", "zipf", "burst")), act=rng.choice(ACTS), bias=rng.random() < 0.5,
                        operand=rng.choice(("none", "add", "mul")))


def _counts(case, seed):
    """Rows of each expert: E whole numbers that sum to P."""
    P, E, r = case["P"], case["E"], np.random.RandomState(seed % (1 << 32))
    if case["skew"] == "spread":                                     # the picks of one token: distinct experts
        c = np.zeros(E, np.int64)
        c[r.permutation(E)[:P]] = 1
        return c
    p = np.full(E, 1.0)
    if case["skew"] == "zipf":
        p = (r.permutation(E) + 1.0) ** -1.1
    elif case["skew"] == "burst":                                    # a tenth of the tokens of 8 picks share an expert
        p[r.randint(E)] += 0.0125 * E
    return r.multinomial(P, p / p.sum())


# --------------------------------------------------------------------------------------------------------- inputs

def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape, dtype=torch.float32, scale=1.0):
        t = torch.empty(*shape, dtype=dtype, device=dev)
        t.normal_(0.0, scale, generator=g)
        return t

    s = {"case": dict(case)}
    if case["op"] in ("route", "train"):
        T, E, K = case["T"], case["E"], case["K"]
        logits = normal(T, E, scale=1.5) + normal(E, scale=0.7)       # tokens differ, some experts are liked by all
        if case["masked"]:
            logits[torch.rand(T, generator=g, device=dev) < case["masked"]] = -math.inf              # padding tokens
            logits[:, torch.rand(E, generator=g, device=dev) < case["masked"]] = -math.inf           # experts out of service
        s["logits"] = logits.to(torch.bfloat16) if case["dtype"] == "bf16" else logits
        s["bias"] = normal(E, scale=0.1) if case["bias"] else None
        if case["op"] == "train":
            s["d_weights"] = normal(T, K)
            s["d_loss"] = torch.ones(1, device=dev)
            s["coef"] = 0.01
        return s
    P, H, N, E, bf = case["P"], case["H"], case["N"], case["E"], torch.bfloat16
    off = np.concatenate([[0], np.cumsum(_counts(case, seed))])
    s["offsets"] = torch.from_numpy(off.astype(np.int32)).to(dev)
    s["segments"] = [int(v) for v in off]
    s["x"] = normal(P, H, dtype=bf)
    s["weight"] = normal(E, N, H, dtype=bf, scale=H ** -0.5)
    s["operand"] = normal(P, N, dtype=bf) if case["operand"] != "none" else None
    if case["op"] == "experts":
        s["bias"] = normal(E, N, dtype=bf, scale=0.1) if case["bias"] else None
    else:
        s["pre"] = normal(P, N, dtype=bf)
        s["dy"] = normal(P, N, dtype=bf)
    return s


# ----------------------------------------------------------------------------------------------------- plain forms

def _plain_scores(logits, scoring):
    """(scores, probabilities that sum to one over a token's experts), 0 where an expert is masked."""
    live = logits > -math.inf
    if scoring == "softmax":
        top = torch.where(live, logits, torch.finfo(torch.float32).min).amax(1, keepdim=True)
        e = torch.where(live, torch.exp(logits - top), 0.0)
        p = e / torch.clamp(e.sum(1, keepdim=True), min=1e-30)
        return p, p
    sg = torch.where(live, 1.0 / (1.0 + torch.exp(-logits)), 0.0)
    return sg, sg / torch.clamp(sg.sum(1, keepdim=True), min=1e-30)


def _plain_route(s):
    c, logits = s["case"], s["logits"].float()
    scores, probs = _plain_scores(logits, c["scoring"])
    key = logits if s["bias"] is None else torch.where(logits > -math.inf, scores + s["bias"], -math.inf)
    key, order = torch.sort(key, dim=1, descending=True, stable=True)
    order, some = order[:, :c["K"]], key[:, :c["K"]] > -math.inf
    picked = torch.where(some, torch.gather(scores, 1, order), 0.0)
    w = picked / torch.clamp(picked.sum(1, keepdim=True), min=1e-30) if c["renorm"] else picked
    return torch.where(some, order, -1).to(torch.int32), w * c["scale"], scores, probs, picked, order, some


def _plain_train(s):
    c, E = s["case"], s["case"]["E"]
    idx, w, scores, probs, picked, order, some = _plain_route(s)
    token = some.any(1, keepdim=True)
    counts = torch.zeros(E, dtype=torch.int32, device=idx.device)
    counts.index_add_(0, order.reshape(-1), some.reshape(-1).to(torch.int32))
    tokens = torch.clamp(token.sum(), min=1).float()
    f = counts.float() * (E / torch.clamp(counts.sum(), min=1).float())
    mean = torch.where(token, probs, 0.0).sum(0) / tokens
    loss = s["coef"] * (f * mean).sum()
    # gradient of the loss with respect to the probabilities, of the weights with respect to the picked scores
    g = s["d_loss"] * s["coef"] / tokens * f
    dbal = probs * (g - (probs * g).sum(1, keepdim=True))
    dw = torch.where(some, s["d_weights"] * c["scale"], 0.0)
    if c["renorm"]:
        total = torch.clamp(picked.sum(1, keepdim=True), min=1e-30)
        dw = (dw - (dw * picked).sum(1, keepdim=True) / total) / total
    dw = torch.where(some, dw, 0.0)
    dscore = torch.zeros_like(scores).scatter_add_(1, order, dw)
    if c["scoring"] == "softmax":
        d = dbal + scores * (dscore - (dscore * scores).sum(1, keepdim=True))
    else:
        d = (dbal + scores * dscore) * (1.0 - scores)
    d = torch.where(token & (scores > 0.0), d, 0.0)
    return {"topk_idx": idx, "topk_weights": w, "counts": counts, "mean_probs": mean, "loss": loss.reshape(1), "dlogits": d.to(s["logits"].dtype)}


def _plain_act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, 0.0)
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return z


def _plain_slope(z, act):
    if act == "relu":
        return (z > 0).float()
    if act == "silu":
        sg = 1.0 / (1.0 + torch.exp(-z))
        return sg * (1.0 + z * (1.0 - sg))
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    return torch.ones_like(z)


def _plain_experts(s):
    # one product an expert: the segments differ in length, and a product padded to the longest costs several times this
    c, seg = s["case"], s["segments"]
    y = torch.empty(c["P"], c["N"], dtype=torch.bfloat16, device=s["x"].device)
    for e in range(c["E"]):
        a, b = seg[e], seg[e + 1]
        if a < b:
            z = s["x"][a:b].float() @ s["weight"][e].float().t()
            if s["bias"] is not None:
                z = z + s["bias"][e].float()
            v = _plain_act(z, c["act"])
            if c["operand"] != "none":
                r = s["operand"][a:b].float()
                v = v + r if c["operand"] == "add" else v * r
            y[a:b] = v
    return {"y": y}


def _plain_backward(s):
    c, seg, bf = s["case"], s["segments"], torch.bfloat16
    out = {"dx": torch.empty_like(s["x"]), "dweight": torch.zeros_like(s["weight"])}
    if c["bias"]:
        out["dbias"] = torch.zeros(c["E"], c["N"], device=s["x"].device)
    z, g = s["pre"].float(), s["dy"].float()
    if c["operand"] == "mul":
        out["doperand"] = (g * _plain_act(z, c["act"])).to(bf)
        g = g * s["operand"].float()
    dz = g * _plain_slope(z, c["act"])
    for e in range(c["E"]):
        a, b = seg[e], seg[e + 1]
        if a < b:
            out["dx"][a:b] = dz[a:b] @ s["weight"][e].float()
            out["dweight"][e] = dz[a:b].t() @ s["x"][a:b].float()
            if c["bias"]:
                out["dbias"][e] = dz[a:b].sum(0)
    return out


# ------------------------------------------------------------------------------------------------------------ run

def _own_buffers(s):
    """What a program allocates once for a shape and keeps: outputs and workspaces."""
    from paper_2609_40093_b200 import ep
    c = s["case"]
    if c["op"] in ("route", "train"):
        s["router"] = ep.Router(c["E"], c["K"], scoring=ep.SCORE_SOFTMAX if c["scoring"] == "softmax" else ep.SCORE_SIGMOID, renormalize=c["renorm"],
                                scale=c["scale"], balance_coef=s.get("coef", 0.0))
        s["routing"] = ep.alloc_routing(c["T"], c["E"], c["K"], balance=c["op"] == "train")
        s["dlogits"] = torch.empty_like(s["logits"])
    else:
        act = {"none": ep.ACT_NONE, "relu": ep.ACT_RELU, "silu": ep.ACT_SILU, "gelu": ep.ACT_GELU}[c["act"]]
        s["how"] = dict(activation=act, operand=s["operand"], operand_op=ep.OPERAND_MUL if c["operand"] == "mul" else ep.OPERAND_ADD)
        if c["op"] == "experts":
            s["y"] = torch.empty(c["P"], c["N"], dtype=torch.bfloat16, device="cuda")
        else:
            s["grads"] = ep.alloc_expert_grads(c["P"], c["H"], c["N"], c["E"], bias=c["bias"], operand=c["operand"] == "mul")
    s["ready"] = True
    return s


def _own_run(s):
    from paper_2609_40093_b200 import ep
    c = s["case"]
    if "ready" not in s:
        _own_buffers(s)
    if c["op"] == "route":
        r = ep.ep_route(s["logits"], s["router"], bias=s["bias"], out=s["routing"])
        return {"topk_idx": r.topk_idx, "topk_weights": r.topk_weights}
    if c["op"] == "train":
        r = ep.ep_route(s["logits"], s["router"], bias=s["bias"], out=s["routing"])
        ep.ep_route_backward(s["logits"], s["router"], r, d_weights=s["d_weights"], d_loss=s["d_loss"], dlogits=s["dlogits"])
        return {"topk_idx": r.topk_idx, "topk_weights": r.topk_weights, "counts": r.expert_counts, "mean_probs": r.mean_probs, "loss": r.loss, "dlogits": s["dlogits"]}
    if c["op"] == "experts":
        return {"y": ep.ep_expert_matmul(s["x"], s["offsets"], s["weight"], bias=s["bias"], y=s["y"], **s["how"])}
    gr = ep.ep_expert_matmul_backward(s["dy"], s["x"], s["offsets"], s["weight"], pre=s["pre"], grads=s["grads"], **s["how"])
    out = {"dx": gr.dx, "dweight": gr.dweight}
    if c["bias"]:
        out["dbias"] = gr.dbias
    if c["operand"] == "mul":
        out["doperand"] = gr.doperand
    return out


def run(state):
    if own:
        return _own_run(state)
    op = state["case"]["op"]
    if op == "route":
        idx, w = _plain_route(state)[:2]
        return {"topk_idx": idx, "topk_weights": w}
    return {"train": _plain_train, "experts": _plain_experts, "backward": _plain_backward}[op](state)


# ----------------------------------------------------------------------------------------------------------- work

def work(case):
    if case["op"] in ("route", "train"):
        T, E, K = case["T"], case["E"], case["K"]
        b = 4 if case["dtype"] == "f32" else 2
        bytes_, flops = T * E * b + T * K * 8 + (4 * E if case["bias"] else 0), 8 * T * E
        if case["op"] == "train":                                   # the logits are read again by the gradient, which is a pass of its own
            bytes_, flops = bytes_ + 2 * T * E * b + T * K * 12 + 16 * E, 24 * T * E
        return {"bytes": bytes_, "flops": flops}
    P, H, N, E = case["P"], case["H"], case["N"], case["E"]
    active = int((_counts(case, 0) > 0).sum())
    if case["op"] == "experts":
        return {"bytes": 2 * (P * H + active * H * N + P * N * (2 if case["operand"] != "none" else 1) + (active * N if case["bias"] else 0)) + 4 * (E + 1),
                "flops": 2 * P * H * N}
    return {"bytes": 2 * (2 * P * H + active * H * N + E * H * N + P * N * (4 if case["operand"] == "mul" else 2)) + (4 * E * N if case["bias"] else 0) + 4 * (E + 1),
            "flops": 4 * P * H * N}


# ---------------------------------------------------------------------------------------------------- in 64 bits

def _exact_route(s, c):
    x = s["logits"].double()
    T, E, K = c["T"], c["E"], c["K"]
    dead = torch.isneginf(x)
    empty = dead.all(1)
    if c["scoring"] == "softmax":
        score = torch.exp(x - torch.logsumexp(x.masked_fill(empty[:, None], 0.0), 1, keepdim=True)).masked_fill(dead, 0.0)
        prob = score
    else:
        score = torch.sigmoid(x).masked_fill(dead, 0.0)
        prob = score / score.sum(1, keepdim=True).masked_fill(empty[:, None], 1.0)
    value = (x if s["bias"] is None else score + s["bias"].double()).masked_fill(dead, -math.inf)
    rank = torch.argsort(torch.argsort(-value, dim=1, stable=True), dim=1)          # place of each expert in its token's order
    pick = (rank < K) & ~dead
    chosen = torch.zeros(T, K + 1, dtype=torch.float64, device=x.device).scatter_(1, torch.where(pick, rank, K), torch.where(pick, score, 0.0))[:, :K]
    ids = torch.full((T, K + 1), -1, dtype=torch.int32, device=x.device)
    ids.scatter_(1, torch.where(pick, rank, K), torch.arange(E, dtype=torch.int32, device=x.device).expand(T, E))
    total = chosen.sum(1, keepdim=True) if c["renorm"] else torch.ones(T, 1, dtype=torch.float64, device=x.device)
    return score, prob, rank, pick, ids[:, :K], chosen / total.masked_fill(total == 0, 1.0) * c["scale"], total, empty


def _exact_train(s, c):
    score, prob, rank, pick, ids, w, total, empty = _exact_route(s, c)
    counts = pick.sum(0)
    n = max(1, int((~empty).sum()))
    f = counts.double() * c["E"] / max(1, int(counts.sum()))
    mean = prob.sum(0) / n
    up = torch.where(pick, torch.gather(s["d_weights"].double(), 1, rank.clamp(max=c["K"] - 1)), 0.0) * c["scale"]     # at each picked expert
    if c["renorm"]:
        t = total.masked_fill(total == 0, 1.0)
        up = torch.where(pick, up / t - (up * torch.where(pick, score, 0.0)).sum(1, keepdim=True) / t ** 2, 0.0)
    gf = (s["d_loss"].double() * s["coef"] / n) * f
    inner = gf - (prob * gf).sum(1, keepdim=True)
    if c["scoring"] == "softmax":
        d = prob * inner + score * up - score * (score * up).sum(1, keepdim=True)
    else:
        d = prob * inner * (1 - score) + score * (1 - score) * up
    return {"topk_idx": None, "topk_weights": w, "counts": None, "mean_probs": mean, "loss": (s["coef"] * (f * mean).sum()).reshape(1), "dlogits": d}


def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["op"] == "route":
        return {"topk_idx": None, "topk_weights": _exact_route(s, c)[5]}
    if c["op"] == "train":
        return _exact_train(s, c)
    fn = {"none": lambda z: z, "relu": torch.relu, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu}[c["act"]]
    seg, d64 = s["segments"], dict(dtype=torch.float64, device="cuda")
    if c["op"] == "experts":
        y = torch.empty(c["P"], c["N"], **d64)
        for e in range(c["E"]):
            rows = slice(seg[e], seg[e + 1])
            z = torch.mm(s["x"][rows].double(), s["weight"][e].double().t())
            v = fn(z if s["bias"] is None else z + s["bias"][e].double())
            y[rows] = v if c["operand"] == "none" else v + s["operand"][rows].double() if c["operand"] == "add" else v * s["operand"][rows].double()
        return {"y": y}
    z = s["pre"].double().requires_grad_(True)
    r = s["operand"].double().requires_grad_(True) if c["operand"] == "mul" else None
    (fn(z) if r is None else fn(z) * r).backward(s["dy"].double())
    out = {"dx": torch.empty(c["P"], c["H"], **d64), "dweight": torch.empty(c["E"], c["N"], c["H"], **d64)}
    if c["bias"]:
        out["dbias"] = torch.empty(c["E"], c["N"], **d64)
    if r is not None:
        out["doperand"] = r.grad
    for e in range(c["E"]):
        rows = slice(seg[e], seg[e + 1])
        torch.mm(z.grad[rows], s["weight"][e].double(), out=out["dx"][rows])
        torch.mm(z.grad[rows].t(), s["x"][rows].double(), out=out["dweight"][e])
        if c["bias"]:
            out["dbias"][e] = z.grad[rows].sum(0)
    return out
