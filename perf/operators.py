"""What is measured of the operators that learn and serve vectors: the path in front of and beside a k-NN graph.

The rows that ``knn_build`` indexes are learnt: ids are looked up in a table, normed with the residual's addition, and scored
against every row of the table by a softmax cross entropy whose gradients come back to the table.  They are served in 8 bits: normed
rows are quantised with a scale each and scored by an integer product.

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
EPS = 1e-6


def listed():
    return [
        # the rows of one request, from the table of the set the library is quoted on: latency counts
        dict(name="lookup_request", op="lookup", n=64, v=1_000_000, d=128, t="fp32"),
        # the gradient of a training step's lookup: few ids take most of the tokens, every row of the table is written
        dict(name="lookup_grad_step", op="lookup_grad", n=65_536, v=131_072, d=1024, t="bf16"),
        # a small set of odd sizes in the library's own type
        dict(name="lookup_grad_odd", op="lookup_grad", n=20_011, v=37_511, d=50, t="fp32"),
        # one request of a serving loop: a few tokens, norm and 8-bit rows
        dict(name="norm_q8_request", op="norm_q8", n=4, d=4096, t="fp16"),
        # a long prompt, or rows made ready for an index
        dict(name="norm_q8_long", op="norm_q8", n=16_384, d=4096, t="bf16"),
        # a training step's norm, there and back, at a descriptor's length and an odd number of rows
        dict(name="norm_step", op="norm_step", n=30_011, d=960, t="bf16"),
        # the same few tokens against a large matrix: its bytes count
        dict(name="product_request", op="product", m=4, n=16_384, k=4096, t="fp16", bias=True),
        # a long prompt: the operations count
        dict(name="product_long", op="product", m=8192, n=8192, k=4096, t="bf16", bias=False),
        # queries scored against every row of an index in 8 bits: the scores' bytes count
        dict(name="product_scores", op="product", m=203, n=1_000_000, k=128, t="fp32", bias=False),
        # the losses of a request's tokens: every row of the table is read once
        dict(name="loss_request", op="loss", n=48, v=131_072, d=1024, t="bf16"),
        # the largest: a training step's loss and both gradients over a large table
        dict(name="loss_step", op="loss_step", n=8192, v=131_072, d=1024, t="bf16"),
        # the same in the library's own type and at odd sizes
        dict(name="loss_step_odd", op="loss_step", n=1_003, v=37_511, d=96, t="fp32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _length(rng, lo, hi):
    """A row length: mostly multiples of 8, some odd ones."""
    d = _log_int(rng, lo, hi)
    return d if rng.random() < 0.25 else max(8, (d + 4) // 8 * 8)


def draw(rng):
    op = rng.choice(["lookup", "lookup_grad", "norm_q8", "norm_step", "product", "product", "loss", "loss_step", "loss_step"])
    t = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if op in ("lookup", "lookup_grad"):
        return dict(op=op, n=_log_int(rng, 1, 131_072), v=_log_int(rng, 500, 262_144), d=_length(rng, 32, 1024), t=t)
    if op in ("norm_q8", "norm_step"):
        return dict(op=op, n=_log_int(rng, 1, 32_768), d=_length(rng, 32, 8192), t=t)
    if op == "product":
        while True:
            c = dict(op=op, m=_log_int(rng, 1, 8192), n=_log_int(rng, 64, 1_000_000), k=_length(rng, 32, 8192), t=t, bias=rng.random() < 0.5)
            if c["m"] * c["n"] <= 1 << 28 and c["m"] * c["n"] * c["k"] <= 1 << 38 and c["n"] * c["k"] <= 1 << 30:
                return c
    while True:
        c = dict(op=op, n=_log_int(rng, 1, 8192), v=_log_int(rng, 500, 131_072), d=_length(rng, 32, 2048), t=t)
        if c["n"] * c["v"] * c["d"] <= (1 << 40 if t != "fp32" else 1 << 37):
            return c


def _popular(gen, n, v):
    """n row numbers below v, the i-th most frequent one about 1 / i of the time, spread over the table."""
    rank = torch.exp(torch.rand(n, generator=gen, device=DEV, dtype=torch.float64) * math.log(v + 1)).long().clamp_(1, v) - 1
    return (rank * 2_654_435_761) % v


def _rows(gen, n, d, t):
    """Activations: normal values, a few channels ten times as large."""
    x = torch.randn(n, d, generator=gen, device=DEV)
    x[:, :: max(1, d // 4)] *= 10.0
    return x.to(t)


def _codes(gen, n, d):
    """8-bit rows with a scale each, as quantising normal rows gives them."""
    x = torch.randn(n, d, generator=gen, device=DEV)
    s = x.abs().amax(1) / 127
    return torch.round(x / s[:, None]).to(torch.int8), s * (0.5 + torch.rand(n, generator=gen, device=DEV))


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    op, t = case["op"], TYPES[case["t"]]
    s = dict(case)
    if op == "product":
        s["a"], s["a_scale"] = _codes(gen, case["m"], case["k"])
        s["b"], s["b_scale"] = _codes(gen, case["n"], case["k"])
        s["add"] = torch.randn(case["n"], generator=gen, device=DEV) if case["bias"] else None
        return s
    n, d = case["n"], case["d"]
    if op in ("lookup", "lookup_grad"):
        v = case["v"]
        ids = _popular(gen, n, v)
        if n > 8:
            ids[torch.randint(0, n, (n // 50,), generator=gen, device=DEV)] = -1      # padding
        s["ids"] = ids
        s["scale"] = math.sqrt(d)
        if op == "lookup":
            s["table"] = (torch.randn(v, d, generator=gen, device=DEV) / math.sqrt(d)).to(t)
        else:
            s["grad"] = torch.randn(n, d, generator=gen, device=DEV).to(t)
        return s
    if op in ("norm_q8", "norm_step"):
        s["x"], s["residual"] = _rows(gen, n, d, t), _rows(gen, n, d, t)
        s["weight"] = (1 + 0.1 * torch.randn(d, generator=gen, device=DEV)).to(t)
        if op == "norm_step":
            s["dy"] = torch.randn(n, d, generator=gen, device=DEV).to(t)
            s["dr"] = torch.randn(n, d, generator=gen, device=DEV).to(t)
        return s
    v = case["v"]
    w = torch.randn(v, d, generator=gen, device=DEV) / math.sqrt(d)
    targets = _popular(gen, n, v)
    # a model on its way: rows lean towards their target
    h = torch.randn(n, d, generator=gen, device=DEV) + 5.0 * torch.rand(n, 1, generator=gen, device=DEV) * w[targets]
    if n > 8:
        targets[torch.randint(0, n, (n // 50,), generator=gen, device=DEV)] = -1      # tokens that are not learnt from
    s["h"], s["w"], s["targets"], s["scale"] = h.to(t), w.to(t), targets, 1.25
    # the weights of the tokens; narrow gradients are formed under a loss scale
    s["dloss"] = (0.5 + torch.rand(n, generator=gen, device=DEV)) / n * (4096.0 if case["t"] == "fp16" else 1.0)
    return s


def _plain_norm(x, residual, eps):
    r = (x.float() + residual.float()).to(x.dtype)
    z = r.float()
    return r, z, torch.rsqrt((z * z).mean(1, keepdim=True) + eps)


def _plain(s):
    op = s["op"]
    if op == "lookup":
        there = (s["ids"] >= 0) & (s["ids"] < s["v"])
        rows = s["table"][s["ids"].clamp(0, s["v"] - 1)].float() * s["scale"]
        return torch.where(there[:, None], rows, 0.0).to(s["table"].dtype)
    if op == "lookup_grad":
        there = (s["ids"] >= 0) & (s["ids"] < s["v"])
        rows = torch.where(there[:, None], s["grad"].float(), 0.0)
        out = torch.zeros(s["v"], s["d"], device=rows.device).index_add_(0, s["ids"].clamp(0, s["v"] - 1), rows)
        return (out * s["scale"]).to(s["grad"].dtype)
    if op == "norm_q8":
        # a value next to a border of the grid falls on one side of it: 64 bits
        r = (s["x"].float() + s["residual"].float()).to(s["x"].dtype)
        z = r.double()
        y = z * torch.rsqrt((z * z).mean(1, keepdim=True) + EPS) * s["weight"].double()
        scale = (y.abs().amax(1) / 127).float()
        q = torch.round(y / scale.double()[:, None]).to(torch.int8)
        return (q.float() * scale[:, None]).to(r.dtype), scale, r
    if op == "norm_step":
        r, z, rstd = _plain_norm(s["x"], s["residual"], EPS)
        w, dy = s["weight"].float(), s["dy"].float()
        y = z * rstd * w
        u = dy * w
        dx = s["dr"].float() + rstd * (u - z * rstd * rstd * (u * z).mean(1, keepdim=True))
        dw = (dy * z * rstd).sum(0)
        return y.to(r.dtype), r, dx.to(r.dtype), dw.to(r.dtype)
    if op == "product":
        # whole numbers up to 127^2 k: exact in 32 bits up to k = 1040, in 64 beyond
        wide = torch.float32 if s["k"] <= 1040 else torch.float64
        out = (s["a"].to(wide) @ s["b"].to(wide).t()).float()
        out = out * s["a_scale"][:, None] * s["b_scale"][None, :]
        if s["add"] is not None:
            out = out + s["add"][None, :]
        return out.to(TYPES[s["t"]])
    h, w, targets = s["h"].float(), s["w"].float(), s["targets"]
    there = (targets >= 0) & (targets < s["v"])
    at = targets.clamp(0, s["v"] - 1)[:, None]
    z = (h @ w.t()) * s["scale"]
    lse = torch.logsumexp(z, 1)
    loss = torch.where(there, lse - z.gather(1, at)[:, 0], 0.0)
    if op == "loss":
        return loss
    g = torch.where(there, s["dloss"], 0.0) * s["scale"]
    p = torch.exp(z - lse[:, None])
    p.scatter_add_(1, at, torch.full_like(at, -1, dtype=p.dtype))
    p = p * g[:, None]
    return loss, (p @ w).to(s["h"].dtype), (p.t() @ h).to(s["w"].dtype)


def run(state):
    s = state
    if not own:
        return _plain(s)
    from paper_2508_08744_amd import embed
    op = s["op"]
    if op == "lookup":
        return embed.lookup(s["table"], s["ids"], scale=s["scale"])
    if op == "lookup_grad":
        return embed.lookup_grad(s["grad"], s["ids"], s["v"], scale=s["scale"])
    if op == "norm_q8":
        q, scale, r = embed.add_rms_norm_q8(s["x"], s["weight"], residual=s["residual"], eps=EPS)
        return embed.dequantize_rows(q, scale, s["x"].dtype), scale, r
    if op == "norm_step":
        y, r, rstd = embed.add_rms_norm(s["x"], s["weight"], residual=s["residual"], eps=EPS)
        dx, dw = embed.add_rms_norm_grad(s["dy"], r, s["weight"], rstd, dr=s["dr"])
        return y, r, dx, dw
    if op == "product":
        return embed.matmul_q8(s["a"], s["a_scale"], s["b"], s["b_scale"], bias=s["add"], out_dtype=TYPES[s["t"]])
    loss, lse = embed.softmax_xent(s["h"], s["w"], s["targets"], scale=s["scale"])
    if op == "loss":
        return loss
    dh, dw = embed.softmax_xent_grad(s["h"], s["w"], s["targets"], lse, s["dloss"], scale=s["scale"])
    return loss, dh, dw


def work(case):
    op, e = case["op"], BYTES[case["t"]]
    if op == "product":
        m, n, k = case["m"], case["n"], case["k"]
        return dict(bytes=(m + n) * (k + 4) + (4 * n if case["bias"] else 0) + m * n * e, flops=2 * m * n * k)
    n, d = case["n"], case["d"]
    if op == "lookup":
        return dict(bytes=2 * n * d * e + 8 * n, flops=n * d)
    if op == "lookup_grad":
        return dict(bytes=(n + case["v"]) * d * e + 8 * n, flops=2 * n * d)
    if op == "norm_q8":
        # the 8-bit rows are written, read back and written as the values they stand for
        return dict(bytes=n * d * (3 * e + 2 + e) + d * e + 4 * n, flops=8 * n * d)
    if op == "norm_step":
        return dict(bytes=n * d * 8 * e + 3 * d * e + 8 * n, flops=16 * n * d)
    v = case["v"]
    if op == "loss":
        return dict(bytes=(n + v) * d * e + 16 * n, flops=2 * n * v * d)
    return dict(bytes=3 * (n + v) * d * e + 32 * n, flops=6 * n * v * d)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "product":
        out = torch.matmul(s["a"].double(), s["b"].double().transpose(0, 1))
        out.mul_(s["a_scale"].double().unsqueeze(1)).mul_(s["b_scale"].double())
        return out if s["add"] is None else out.add_(s["add"].double())
    if op == "lookup":
        out = torch.zeros(case["n"], case["d"], dtype=torch.float64, device=DEV)
        at = torch.nonzero(s["ids"] >= 0).squeeze(1)
        out[at] = torch.index_select(s["table"], 0, s["ids"][at]).double() * s["scale"]
        return out
    if op == "lookup_grad":
        at = torch.nonzero(s["ids"] >= 0).squeeze(1)
        order = torch.argsort(s["ids"][at], stable=True)
        run_ids, counts = torch.unique_consecutive(s["ids"][at][order], return_counts=True)
        out = torch.zeros(case["v"], case["d"], dtype=torch.float64, device=DEV)
        if at.numel():
            # sums over runs of the sorted tokens: differences of a running sum, which 64 bits carry
            total = torch.cumsum(s["grad"][at][order].double(), 0)
            ends = total[torch.cumsum(counts, 0) - 1]
            out[run_ids] = torch.diff(ends, dim=0, prepend=torch.zeros_like(ends[:1])) * s["scale"]
        return out
    if op in ("norm_q8", "norm_step"):
        # the residual stream is kept in the inputs' type: its rounding is part of the definition
        r = (s["x"].double() + s["residual"].double()).to(s["x"].dtype).double()
        size = torch.sqrt(torch.linalg.vecdot(r, r) / case["d"] + EPS).unsqueeze(1)
        unit = r / size
        y = unit * s["weight"].double()
        if op == "norm_q8":
            step = (torch.linalg.vector_norm(y, ord=float("inf"), dim=1) / 127).float().double()
            return torch.round(y / step.unsqueeze(1)) * step.unsqueeze(1), step, r
        dy = s["dy"].double()
        u = dy * s["weight"].double()
        # the norm's Jacobian: what of u is across r, over r's size
        along = torch.linalg.vecdot(u, unit).unsqueeze(1) / case["d"]
        return y, r, s["dr"].double() + (u - unit * along) / size, torch.linalg.vecdot(dy, unit, dim=0)
    # the table in pieces, running maximum and sum, then the gradients of each piece
    h, n, v, c = s["h"].double(), case["n"], case["v"], s["scale"]
    t, there = s["targets"], s["targets"] >= 0
    step = max(1, (1 << 27) // n)
    pieces = [(i, s["w"][i:i + step].double()) for i in range(0, v, step)]
    top = torch.full((n,), -math.inf, dtype=torch.float64, device=DEV)
    mass = torch.zeros_like(top)
    for _, w in pieces:
        z = c * torch.matmul(h, w.transpose(0, 1))
        new = torch.maximum(top, z.amax(1))
        mass = mass * torch.exp(top - new) + torch.exp(z - new.unsqueeze(1)).sum(1)
        top = new
    lse = top + torch.log(mass)
    rows = s["w"][t.clamp_min(0)].double()
    loss = torch.where(there, lse - c * torch.linalg.vecdot(h, rows), torch.zeros_like(lse))
    if op == "loss":
        return loss
    g = torch.where(there, s["dloss"].double(), torch.zeros_like(lse)) * c
    dh = -g.unsqueeze(1) * rows
    dw = torch.zeros(v, case["d"], dtype=torch.float64, device=DEV)
    for i, w in pieces:
        p = torch.exp(c * torch.matmul(h, w.transpose(0, 1)) - lse.unsqueeze(1)) * g.unsqueeze(1)
        dh += torch.matmul(p, w)
        dw[i:i + len(w)] = torch.matmul(p.transpose(0, 1).contiguous(), h)
    at = torch.nonzero(there).squeeze(1)
    dw.index_add_(0, t[at], -g[at].unsqueeze(1) * h[at])
    return loss, dh, dw
