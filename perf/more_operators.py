"""What is measured of the operators that tune a learnt table by what it answers with, and of those between its gradients and its update.

A table's rows are scored against tokens; a user asks how likely given rows are, how sure the table is (the entropy), and for the rows it
would rather have answered with.  Tuning by rewards takes the gradients of the first two.  Gradients of all tensors are brought under one norm
before the update.

A case names an operator (``op``) and its sizes.  ``listed`` gives the fixed ones, ``draw`` more of the same ranges, ``prepare`` makes a
case's inputs on the GPU from a seed, ``run`` is one pass, ``work`` what a pass cannot do without, ``exact`` the same from the
definition in 64 bits.  With ``own`` false ``run`` is the plain form in elementary torch operations.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}


def listed():
    return [
        # one step of a serving loop: the next row and its alternatives; the table's bytes count
        dict(name="answer_one", op="log_probs", n=1, v=131_072, d=1024, t="bf16", top=8),
        # a few requests over the table of a small set: latency counts
        dict(name="answer_small", op="log_probs", n=4, v=20_000, d=128, t="fp32", top=5),
        # the tokens of many requests at once, as many alternatives as interfaces offer
        dict(name="answer_request", op="log_probs", n=48, v=131_072, d=1024, t="bf16", top=20),
        # a long prompt with alternatives: the operations count
        dict(name="answer_long", op="log_probs", n=4096, v=131_072, d=1024, t="bf16", top=8),
        # held-out tokens scored, without alternatives, at odd sizes
        dict(name="score_odd", op="log_probs", n=2_003, v=50_257, d=500, t="fp16", top=0),
        # the same in the library's own type
        dict(name="score_odd_wide", op="log_probs", n=1_003, v=37_511, d=96, t="fp32", top=3),
        # the largest: a step of tuning by rewards over a large table, with a bonus for the entropy
        dict(name="tune_step", op="tune", n=4096, v=131_072, d=1024, t="bf16", table=True),
        # the table stays as it is, and what is in front of it is tuned
        dict(name="tune_frozen", op="tune", n=999, v=37_511, d=512, t="fp16", table=False),
        # a small set of odd sizes in the library's own type
        dict(name="tune_odd", op="tune", n=301, v=9_001, d=50, t="fp32", table=True),
        # the gradients of a small table and its norm
        dict(name="clip_small", op="clip", v=20_000, d=128, layers=0, t="bf16", clipped=True),
        # those of a large table and of many layers' matrices and weights, formed under a loss scale
        dict(name="clip_model", op="clip", v=131_072, d=1024, layers=60, t="fp16", clipped=True),
        # many small gradients of odd sizes: calls and launches count
        dict(name="norm_many", op="norm", v=1_009, d=33, layers=150, t="fp32", clipped=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _length(rng, lo, hi):
    """A row length: mostly multiples of 8, some odd ones."""
    d = _log_int(rng, lo, hi)
    return d if rng.random() < 0.25 else max(8, (d + 4) // 8 * 8)


def draw(rng):
    op = rng.choice(["log_probs", "log_probs", "log_probs", "tune", "tune", "clip", "clip", "norm"])
    t = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if op in ("clip", "norm"):
        while True:
            c = dict(op=op, v=_log_int(rng, 100, 131_072), d=_length(rng, 16, 1024), layers=rng.choice([0, 1, rng.randint(2, 160)]), t=t,
                     clipped=op == "clip" and rng.random() < 0.8)
            if (c["v"] + c["layers"] * c["d"]) * c["d"] <= 1 << 27:
                return c
    while True:
        c = dict(op=op, n=_log_int(rng, 1, 8192), v=_log_int(rng, 500, 131_072), d=_length(rng, 32, 2048), t=t)
        if op == "log_probs":
            c["top"] = rng.choice([0, 1, 5, 8, 20, rng.randint(2, 32)])
        else:
            c["table"] = rng.random() < 0.7
        if c["n"] * c["v"] <= 1 << 29 and c["n"] * c["v"] * c["d"] <= (1 << 39 if t != "fp32" else 1 << 36):
            return c


def _popular(gen, n, v):
    """n row numbers below v, the i-th most frequent one about 1 / i of the time, spread over the table."""
    rank = torch.exp(torch.rand(n, generator=gen, device=DEV, dtype=torch.float64) * math.log(v + 1)).long().clamp_(1, v) - 1
    return (rank * 2_654_435_761) % v


def _sizes(case):
    """The values of every gradient, and whether it is kept in fp32: the table's, then a matrix and a norm's weight a layer."""
    d = case["d"]
    return [(case["v"] * d, False), (d, True)] + [(d * d, False), (d, True)] * case["layers"]


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    op, t = case["op"], TYPES[case["t"]]
    s = dict(case)
    if op in ("clip", "norm"):
        loss_scale = 4096.0 if case["t"] == "fp16" else 1.0
        sizes = _sizes(case)
        # the whole norm is a few times what it is brought under, or half of it; layers differ
        size = (3.0 if case["clipped"] else 0.5) * loss_scale / math.sqrt(sum(n for n, _ in sizes))
        s["grads"] = [(torch.randn(n, generator=gen, device=DEV) * (size * (0.5 + torch.rand(1, generator=gen, device=DEV)))).to(torch.float32 if wide else t)
                      for n, wide in sizes]
        s["scale"], s["max_norm"] = 1.0 / loss_scale, 1.0
        if op == "clip":
            # where the update reads them: one buffer a type, a tensor behind the other
            s["flat"] = {u: torch.zeros(sum(g.numel() for g in s["grads"] if g.dtype == u), dtype=u, device=DEV) for u in {t, torch.float32}}
            at = dict.fromkeys(s["flat"], 0)
            s["out"] = []
            for g in s["grads"]:
                s["out"].append(s["flat"][g.dtype][at[g.dtype]:at[g.dtype] + g.numel()])
                at[g.dtype] += g.numel()
        return s
    n, v, d = case["n"], case["v"], case["d"]
    w = torch.randn(v, d, generator=gen, device=DEV) / math.sqrt(d)
    targets = _popular(gen, n, v)
    # a model on its way: rows lean towards the given row, some more than others
    h = 2.0 * torch.randn(n, d, generator=gen, device=DEV) + 8.0 * torch.rand(n, 1, generator=gen, device=DEV) * w[targets]
    if n > 8:
        targets[torch.randint(0, n, (n // 50,), generator=gen, device=DEV)] = -1      # padding
    s["h"], s["w"], s["targets"], s["scale"] = h.to(t), w.to(t), targets, 1.25
    if op == "tune":
        # rewards above and below their mean, and the entropy's weight; narrow gradients are formed under a loss scale
        size = (4096.0 if case["t"] == "fp16" else 1.0) / n
        s["dlogp"] = -size * torch.randn(n, generator=gen, device=DEV)
        s["dentropy"] = torch.where(targets >= 0, -0.05 * size, 0.0)
    return s


def _plain_clip(s):
    total = sum((g.float() * g.float()).double().sum() for g in s["grads"])
    norm = (torch.sqrt(total) * abs(s["scale"])).float()
    if s["op"] == "norm":
        return norm
    factor = s["scale"] * torch.clamp(s["max_norm"] / norm, max=1.0)
    wide = [g * factor for g in s["grads"] if g.dtype == torch.float32]
    narrow = [(g.float() * factor).to(g.dtype) for g in s["grads"] if g.dtype != torch.float32]
    return [norm, torch.cat(wide)] + ([torch.cat(narrow)] if narrow else [])


def _plain(s):
    if s["op"] in ("clip", "norm"):
        return _plain_clip(s)
    h, w, targets, top = s["h"], s["w"], s["targets"], s.get("top", 0)
    there = (targets >= 0) & (targets < s["v"])
    at = targets.clamp(0, s["v"] - 1)[:, None]
    if top:
        # two rows whose scores are close change places by a rounding in 32 bits: 64
        best = (h.double() @ w.double().t()) * s["scale"]
        z = best.float()
        best, rows = torch.topk(best, top, dim=1)
    else:
        z = (h.float() @ w.float().t()) * s["scale"]
    lse = torch.logsumexp(z, 1)
    logp = torch.where(there, z.gather(1, at)[:, 0] - lse, 0.0)
    p = torch.exp(z - lse[:, None])
    entropy = lse - (p * z).sum(1)
    if s["op"] == "log_probs":
        return [logp, entropy] + ([rows.int(), (best - lse.double()[:, None]).float()] if top else [])
    a = torch.where(there, s["dlogp"], 0.0)[:, None]
    b = s["dentropy"][:, None]
    p = -p * (a + b * (z - lse[:, None] + entropy[:, None]))
    p = p.scatter_add_(1, at, a) * s["scale"]
    dh = (p @ w.float()).to(h.dtype)
    return [logp, entropy, dh] + ([(p.t() @ h.float()).to(w.dtype)] if s["table"] else [])


def run(state):
    s = state
    if not own:
        return _plain(s)
    from paper_2508_08744_amd import learn
    if s["op"] == "norm":
        return learn.grad_norm(s["grads"], scale=s["scale"])
    if s["op"] == "clip":
        norm = learn.clip_grads(s["grads"], s["max_norm"], scale=s["scale"], out=s["out"])
        return [norm, s["flat"][torch.float32]] + [f for u, f in s["flat"].items() if u != torch.float32]
    logp, entropy, lse, rows, best = learn.log_probs(s["h"], s["w"], s["targets"], scale=s["scale"], top=s.get("top", 0))
    if s["op"] == "log_probs":
        return [logp, entropy] + ([rows, best] if s["top"] else [])
    dh, dw = learn.log_probs_grad(s["h"], s["w"], s["targets"], lse, s["dlogp"], entropy, s["dentropy"], scale=s["scale"], table=s["table"])
    return [logp, entropy, dh] + ([dw] if s["table"] else [])


def work(case):
    op, e = case["op"], BYTES[case["t"]]
    if op in ("clip", "norm"):
        count = sum(n for n, _ in _sizes(case))
        held = sum(n * (4 if wide else e) for n, wide in _sizes(case))
        return dict(bytes=held * (2 if op == "clip" else 1) + 4, flops=count * (3 if op == "clip" else 2))
    n, v, d = case["n"], case["v"], case["d"]
    if op == "log_probs":
        return dict(bytes=(n + v) * d * e + n * (16 + 8 * case["top"]), flops=2 * n * v * d)
    # the logits, and a product for each gradient
    return dict(bytes=(2 * n + v) * d * e + (v * d * e if case["table"] else 0) + 32 * n, flops=(6 if case["table"] else 4) * n * v * d)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op in ("clip", "norm"):
        norm = abs(s["scale"]) * math.hypot(*(torch.linalg.vector_norm(g.double()).item() for g in s["grads"]))
        if op == "norm":
            return torch.tensor(norm, dtype=torch.float64)
        by = s["scale"] * (s["max_norm"] / norm if norm > s["max_norm"] else 1.0)
        kinds = [torch.float32] + ([TYPES[case["t"]]] if case["t"] != "fp32" else [])
        return [torch.tensor(norm, dtype=torch.float64)] + [by * torch.cat([g for g in s["grads"] if g.dtype == u]).double() for u in kinds]
    # the table in pieces: running maximum, sum, and sum of what is below the maximum, with the best rows so far
    h, n, v, c, top = s["h"].double(), case["n"], case["v"], s["scale"], case.get("top", 0)
    t, there = s["targets"], s["targets"] >= 0
    step = max(1, (1 << 27) // n)
    pieces = [(i, s["w"][i:i + step].double()) for i in range(0, v, step)]
    high = torch.full((n,), -math.inf, dtype=torch.float64, device=DEV)
    mass, below = torch.zeros_like(high), torch.zeros_like(high)
    best = torch.empty(n, 0, dtype=torch.float64, device=DEV)
    rows = torch.empty(n, 0, dtype=torch.int64, device=DEV)
    for i, w in pieces:
        z = c * torch.matmul(h, w.transpose(0, 1))
        new = torch.maximum(high, z.amax(1))
        drop = torch.where(torch.isinf(high), torch.zeros_like(high), new - high)
        fall = torch.exp(-drop)
        under = z - new.unsqueeze(1)
        part = torch.exp(under)
        below = (below - drop * mass) * fall + (part * under).sum(1)
        mass = mass * fall + part.sum(1)
        high = new
        if top:
            value, place = torch.topk(z, min(top, z.shape[1]), dim=1)
            best, rows = torch.cat([best, value], 1), torch.cat([rows, place + i], 1)
            best, place = torch.topk(best, min(top, best.shape[1]), dim=1)
            rows = torch.gather(rows, 1, place)
    lse = high + torch.log(mass)
    entropy = torch.log(mass) - below / mass
    mine = s["w"][t.clamp_min(0)].double()
    logp = torch.where(there, c * torch.linalg.vecdot(h, mine) - lse, torch.zeros_like(lse))
    if op == "log_probs":
        return [logp, entropy] + ([rows.int(), best - lse.unsqueeze(1)] if top else [])
    a = torch.where(there, s["dlogp"].double(), torch.zeros_like(lse))
    b = s["dentropy"].double()
    dh = (c * a).unsqueeze(1) * mine
    dw = torch.zeros(v, case["d"], dtype=torch.float64, device=DEV) if case["table"] else None
    for i, w in pieces:
        log_p = c * torch.matmul(h, w.transpose(0, 1)) - lse.unsqueeze(1)
        p = torch.exp(log_p) * (-c * (a.unsqueeze(1) + b.unsqueeze(1) * (log_p + entropy.unsqueeze(1))))
        dh += torch.matmul(p, w)
        if dw is not None:
            dw[i:i + len(w)] = torch.matmul(p.transpose(0, 1).contiguous(), h)
    if dw is None:
        return [logp, entropy, dh]
    at = torch.nonzero(there).squeeze(1)
    dw.index_add_(0, t[at], (c * a[at]).unsqueeze(1) * h[at])
    return [logp, entropy, dh, dw]
