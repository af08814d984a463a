"""The operators of include/tagore_embed.h against plain forms in 64 bits on the CPU.

Tolerances are bounds, from the roundings that a result goes through: half a step of its type, and for every fp32 sum its longest chain
of additions times 2^-24 of the sum of the terms' magnitudes.
"""
import math

import pytest
import torch

from paper_2508_08744_amd import embed, knn

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]
U = 2.0 ** -24


def half_step(t):
    return torch.finfo(t).eps / 2


def gen(seed):
    return torch.Generator().manual_seed(seed)


def near(got, want, bound, t):
    """|got - want| <= bound (of the fp32 work) + the rounding to t."""
    got, want = got.detach().cpu().double(), want.double()
    tol = bound + half_step(t) * (want.abs() + bound) + torch.finfo(t).tiny
    assert torch.isfinite(got).all()
    off = ((got - want).abs() - tol).max().item() if got.numel() else -1.0
    assert off <= 0.0, "beyond the bound by %g" % off


def strided(x, extra, offset=0):
    """The same matrix with rows `extra` elements further apart, from element `offset` of its memory on."""
    n, d = x.shape
    flat = torch.full((offset + n * (d + extra),), float("nan") if x.is_floating_point() else 77, dtype=x.dtype, device=x.device)
    y = flat[offset:].view(n, d + extra)[:, :d]
    y.copy_(x)
    return y


# ---- lookup

@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("n,v,d", [(1, 1, 1), (3, 500, 8), (64, 1000, 128), (257, 37, 50), (1000, 5000, 127), (33, 70, 1031)])
def test_lookup(t, n, v, d):
    g = gen(n + d)
    table = torch.randn(v, d, generator=g).to(t).to(DEV)
    ids = torch.randint(-2, v + 2, (n,), generator=g)
    want = torch.where(((ids >= 0) & (ids < v))[:, None], table.cpu().double()[ids.clamp(0, v - 1)] * 2.75, 0.0)
    for i in (ids, ids.int()):
        near(embed.lookup(table, i.to(DEV), scale=2.75), want, want.abs() * U, t)
    near(embed.lookup(strided(table, 3, 1), ids.to(DEV), scale=2.75), want, want.abs() * U, t)


def test_lookup_shapes_and_far_rows():
    # rows beyond 2^31 elements of the table
    v, d = 34_000_000, 64
    table = torch.empty(v, d, dtype=BF16, device=DEV)
    ids = torch.tensor([[0, v - 1], [v - 2, 17]], device=DEV)
    rows = torch.randn(4, d, generator=gen(1)).to(BF16).to(DEV)
    table[ids.flatten()] = rows
    assert torch.equal(embed.lookup(table, ids), rows.view(2, 2, d))
    assert embed.lookup(table, ids[:0]).shape == (0, 2, d)


GRAD_SHAPES = [(1, 1, 1), (5, 3, 8), (31, 7, 50), (33, 1, 128), (64, 5000, 96), (1000, 37, 127), (4097, 300, 1031), (16_384, 70_000, 16), (16_385, 70_000, 16),
               (20_000, 3, 40), (50_000, 5_000_000, 8)]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("n,v,d", GRAD_SHAPES)
def test_lookup_grad(t, n, v, d):
    g = gen(n + v + d)
    grad = torch.randn(n, d, generator=g).to(t)
    # a few ids take most tokens; some are no rows
    ids = (torch.rand(n, generator=g, dtype=torch.float64) ** 4 * (v + 2)).long() - 1
    there = (ids >= 0) & (ids < v)
    want = torch.zeros(v, d, dtype=torch.float64).index_add_(0, ids[there], grad[there].double()) * 1.5
    mass = torch.zeros(v, d, dtype=torch.float64).index_add_(0, ids[there], grad[there].double().abs()) * 1.5
    bound = mass * (n + 2) * U if n < 2000 else mass * (32 + n / 32 / 4 + 6) * U
    got = embed.lookup_grad(grad.to(DEV), ids.to(DEV), v, scale=1.5)
    near(got, want, bound, t)
    again = embed.lookup_grad(strided(grad.to(DEV), 5, 1), ids.int().to(DEV), v, scale=1.5)
    assert torch.equal(got, again)                       # equal inputs, equal results
    # added to what is there, in fp32 and in the gradient's type; rows without a token are not touched
    base = torch.randn(v, d, generator=g)
    for to in {F32, t}:
        out = base.to(to).to(DEV)
        before = out.clone()
        assert embed.lookup_grad(grad.to(DEV), ids.to(DEV), v, scale=1.5, out=out) is out
        near(out, before.cpu().double() + want, bound + (want.abs() + bound) * U, to)
        still = torch.ones(v, dtype=torch.bool)
        still[ids[there]] = False
        assert torch.equal(out.cpu()[still], before.cpu()[still])


@pytest.mark.parametrize("n", [100, 20_000])
def test_lookup_grad_without_a_token(n):
    ids = torch.full((n,), -1, device=DEV)
    grad = torch.full((n, 33), float("nan"), dtype=BF16, device=DEV)
    assert torch.equal(embed.lookup_grad(grad, ids, 7), torch.zeros(7, 33, dtype=BF16, device=DEV))
    assert torch.equal(embed.lookup_grad(grad[:0], ids[:0], 7), torch.zeros(7, 33, dtype=BF16, device=DEV))


def test_lookup_grad_is_the_lookups_difference():
    g = gen(5)
    table, way, grad = (torch.randn(s, generator=g, dtype=torch.float64) for s in ((40, 24), (40, 24), (300, 24)))
    ids = torch.randint(0, 40, (300,), generator=g)
    eps = 1e-3

    def value(t):
        return ((t[ids] * 3.0) * grad).sum().item()
    got = embed.lookup_grad(grad.float().to(DEV), ids.to(DEV), 40, scale=3.0).cpu().double()
    slope = (value(table + eps * way) - value(table - eps * way)) / (2 * eps)
    size = (torch.zeros(40, 24, dtype=torch.float64).index_add_(0, ids, grad.abs()) * 3.0 * way.abs()).sum().item()
    assert abs((got * way).sum().item() - slope) <= size * 310 * U + 1e-9 * size


# ---- norm

NORM_SHAPES = [(1, 1), (3, 7), (5, 64), (70, 96), (33, 127), (9, 513), (40, 960), (7, 2048), (6, 2050), (5, 4096), (4, 5001), (3, 8192), (2, 8191)]
CHAIN = 64          # additions of the longest chain of a row's sum: 32 in a lane, 6 over a wave, 16 over the waves, and a few roundings


def _norm_ref(x, res, w, eps):
    r = (x.float() + res.float()).to(x.dtype) if res is not None else x
    z = r.double()
    rstd = 1.0 / torch.sqrt((z * z).mean(1, keepdim=True) + eps)
    return r, z, rstd, z * rstd * w.double()


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("n,d", NORM_SHAPES)
def test_norm_and_gradient(t, n, d):
    g = gen(n * d)
    x, res, dy, dr = (torch.randn(n, d, generator=g).to(t) for _ in range(4))
    w = (1 + 0.2 * torch.randn(d, generator=g)).to(t)
    dev = [v.to(DEV) for v in (x, res, dy, dr, w)]
    for residual, dr_in, extra in ((res, dr, 0), (None, None, 3)):
        r, z, rstd, y = _norm_ref(x, residual, w, 1e-5)
        xs = strided(dev[0], extra, extra) if extra else dev[0]
        got_y, got_r, got_rstd = embed.add_rms_norm(xs, dev[4], None if residual is None else dev[1], eps=1e-5)
        assert torch.equal(got_r.cpu(), r)
        near(got_rstd, rstd[:, 0], rstd[:, 0] * CHAIN * U, F32)
        near(got_y, y, y.abs() * (CHAIN + 4) * U, t)
        u = dy.double() * w.double()
        mean, size = (u * z * rstd).mean(1, keepdim=True), (u * z * rstd).abs().mean(1, keepdim=True)
        dx = rstd * (u - z * rstd * mean) + (dr_in.double() if dr_in is not None else 0.0)
        bound = (3 * CHAIN + 8) * U * (rstd * (u.abs() + (z * rstd).abs() * size) + (dr_in.double().abs() if dr_in is not None else 0.0))
        got_dx, got_dw = embed.add_rms_norm_grad(strided(dev[2], extra) if extra else dev[2], got_r, dev[4], got_rstd, dr=None if dr_in is None else dev[3])
        near(got_dx, dx, bound, t)
        terms = dy.double() * z * rstd
        near(got_dw, terms.sum(0), terms.abs().sum(0) * (n + CHAIN + 8) * U, t)


@pytest.mark.parametrize("n,d", [(5000, 96), (3000, 960)])
def test_norm_gradient_of_many_rows(n, d):
    g = gen(n)
    x, dy = torch.randn(n, d, generator=g), torch.randn(n, d, generator=g)
    w = 1 + 0.2 * torch.randn(d, generator=g)
    _, r, rstd = embed.add_rms_norm(x.to(DEV), w.to(DEV))
    dx, dw = embed.add_rms_norm_grad(dy.to(DEV), r, w.to(DEV), rstd)
    z = x.double()
    terms = dy.double() * z / torch.sqrt((z * z).mean(1, keepdim=True) + 1e-6)
    # (rows of a workgroup one after another, then 64 stretches of the parts, then a tree)
    near(dw, terms.sum(0), terms.abs().sum(0) * (CHAIN + n / 1024 + 4096 / 64 + 8) * U, F32)
    dx2, dw2 = embed.add_rms_norm_grad(dy.to(DEV), r, w.to(DEV), rstd)
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2)


def test_norm_gradient_is_the_norms_difference():
    g = gen(8)
    x, res, w, dy, dr, way = (torch.randn(s, generator=g, dtype=torch.float64).float().double() for s in ((6, 40), (6, 40), (40,), (6, 40), (6, 40), (6, 40)))
    way_w = torch.randn(40, generator=g, dtype=torch.float64)

    def value(x, w):
        r = x + res
        return ((r / torch.sqrt((r * r).mean(1, keepdim=True) + 1e-6) * w) * dy).sum().item() + (r * dr).sum().item()
    f = [v.float().to(DEV) for v in (x, res, w, dy, dr)]
    _, r, rstd = embed.add_rms_norm(f[0], f[2], f[1])
    dx, dw = embed.add_rms_norm_grad(f[3], r, f[2], rstd, dr=f[4])
    e = 1e-4
    assert abs((dx.cpu().double() * way).sum().item() - (value(x + e * way, w) - value(x - e * way, w)) / (2 * e)) < 1e-4
    assert abs((dw.cpu().double() * way_w).sum().item() - (value(x, w + e * way_w) - value(x, w - e * way_w)) / (2 * e)) < 1e-4


# ---- 8-bit rows

@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("n,d", NORM_SHAPES)
def test_norm_to_8_bits(t, n, d):
    g = gen(n * d + 1)
    x, res = torch.randn(n, d, generator=g).to(t), torch.randn(n, d, generator=g).to(t)
    x[:, :: max(1, d // 3)] *= 20
    w = (1 + 0.2 * torch.randn(d, generator=g)).to(t)
    for residual in (res, None):
        r, z, rstd, y = _norm_ref(x, residual, w, 1e-6)
        q, scale, got_r = embed.add_rms_norm_q8(strided(x.to(DEV), 1, 1), w.to(DEV), None if residual is None else residual.to(DEV))
        _grid(q, scale, y)
        assert torch.equal(got_r.cpu(), r)
    q, scale = embed.quantize_rows(strided(x.to(DEV), 2, 3))
    _grid(q, scale, x.double())
    for to in TYPES:
        want = q.cpu().double() * scale.cpu().double()[:, None]
        near(embed.dequantize_rows(q, scale, to), want, want.abs() * U, to)


def _grid(q, scale, y):
    """q and scale are y on its grid, except that a value within 1e-9 of a border may be on either side."""
    q, scale = q.cpu().double(), scale.cpu().double()
    top = y.abs().amax(1) / 127
    assert ((scale - top).abs() <= top * 2 * U).all()
    at = torch.where(scale[:, None] > 0, y / scale[:, None], 0.0)
    assert ((at - q).abs() <= 0.5 + 1e-9).all() and (q.abs() <= 127).all()
    assert (q.abs().amax(1) == torch.where(top > 0, 127.0, 0.0)).all()


def test_8_bit_rows_without_a_grid():
    x = torch.ones(5, 70)
    x[0] = 0
    x[1, 69] = float("nan")
    x[2, 0] = float("inf")
    x[3] = 1e-42
    x[3, 3] = 3e-42
    q, scale = embed.quantize_rows(x.to(DEV))
    q, scale = q.cpu(), scale.cpu()
    assert scale[0] == 0 and torch.isnan(scale[1]) and torch.isnan(scale[2]) and (q[:3] == 0).all()
    assert (q[3].abs() <= 127).all() and q[4].eq(127).all()
    y = embed.dequantize_rows(q.to(DEV), scale.to(DEV)).cpu()
    assert (y[0] == 0).all() and torch.isnan(y[1:3]).all()
    w = torch.ones(70, device=DEV)
    q, scale, _ = embed.add_rms_norm_q8(x.to(DEV), w, eps=0.0)
    assert torch.isnan(scale.cpu()[:3]).all() and (q.cpu()[:3] == 0).all()          # (the norm of a row of zeros is not finite without eps)
    q, scale, _ = embed.add_rms_norm_q8(x.to(DEV), w)
    assert scale.cpu()[0] == 0 and q.cpu()[4].eq(127).all()
    x[1:3] = 1
    y, _, _ = embed.add_rms_norm(x.to(DEV), w)
    assert (y.cpu()[0] == 0).all() and torch.isfinite(y).all()


# ---- product

@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 300, 64), (4, 1000, 256), (16, 17, 4096), (17, 100, 50), (33, 257, 129), (64, 130, 1000), (65, 64, 64),
                                   (100, 333, 128), (300, 1000, 200), (129, 65, 4112), (700, 5100, 96)])
def test_product(t, m, n, k):
    g = gen(m + n + k)
    a = torch.randint(-128, 128, (m, k), generator=g, dtype=torch.int8)
    b = torch.randint(-128, 128, (n, k), generator=g, dtype=torch.int8)
    sa, sb, bias = torch.rand(m, generator=g) / 100, torch.rand(n, generator=g) / 100, torch.randn(n, generator=g)
    prod = (a.double() @ b.double().t()) * sa.double()[:, None] * sb.double()
    for add in (None, bias):
        want = prod if add is None else prod + add.double()
        bound = 4 * U * (prod.abs() + (0 if add is None else add.double().abs()))
        got = embed.matmul_q8(a.to(DEV), sa.to(DEV), b.to(DEV), sb.to(DEV), bias=None if add is None else add.to(DEV), out_dtype=t)
        near(got, want, bound, t)
    # from memory that begins at an odd byte
    odd = [torch.empty(x.numel() + 1, dtype=torch.int8, device=DEV)[1:].view(x.shape).copy_(x) for x in (a, b)]
    assert torch.equal(embed.matmul_q8(odd[0], sa.to(DEV), odd[1], sb.to(DEV), bias=bias.to(DEV), out_dtype=t), got)


@pytest.mark.parametrize("m", [7, 130])
def test_product_of_the_largest_sums(m):
    k = 65536
    a = torch.full((m, k), -128, dtype=torch.int8, device=DEV)
    b = torch.full((40, k), -128, dtype=torch.int8, device=DEV)
    one = torch.ones(m, device=DEV), torch.ones(40, device=DEV)
    assert (embed.matmul_q8(a, one[0], b[:, :].clone(), one[1]) == 2.0 ** 30).all()
    b.fill_(127)
    assert (embed.matmul_q8(a, one[0], b, one[1]) == -128.0 * 127 * k).all()


def test_product_of_far_rows():
    # the output passes 2^31 elements, the weight 2^31 bytes
    n, k = 17_000_000, 128
    b = torch.randint(-128, 128, (n, k), dtype=torch.int8, device=DEV)
    a = torch.randint(-128, 128, (130, k), dtype=torch.int8, device=DEV)
    sa, sb = torch.rand(130, device=DEV), torch.rand(n, device=DEV)
    at = torch.tensor([0, 1, 8_388_607, 8_388_608, 16_777_216, n - 1], device=DEV)
    want = (a.double() @ b[at].double().t()) * sa.double()[:, None] * sb[at].double()
    for m in (3, 130):
        got = embed.matmul_q8(a[:m].contiguous(), sa[:m].contiguous(), b, sb, out_dtype=BF16)
        near(got[:, at], want[:m].cpu(), want[:m].cpu().abs() * 4 * U, BF16)


# ---- softmax cross entropy

XENT_SHAPES = [(1, 1, 1), (2, 3, 8), (1, 700, 64), (30, 129, 96), (33, 1000, 50), (64, 257, 128), (65, 300, 40), (130, 515, 33), (300, 2100, 72), (257, 8000, 130)]


def _xent_inputs(t, n, v, d, seed, ignored=True):
    g = gen(seed)
    w = (torch.randn(v, d, generator=g) / math.sqrt(d)).to(t)
    targets = torch.randint(0, v, (n,), generator=g)
    h = (torch.randn(n, d, generator=g) + 3 * w[targets].float()).to(t)
    if ignored and n > 2:
        targets[::7] = -1
        targets[3::31] = v
    return h, w, targets, 0.5 + torch.rand(n, generator=g)


def _xent_ref(h, w, targets, dloss, scale):
    v = w.shape[0]
    there = (targets >= 0) & (targets < v)
    at = targets.clamp(0, v - 1)[:, None]
    z = (h.double() @ w.double().t()) * scale
    lse = torch.logsumexp(z, 1)
    loss = torch.where(there, lse - z.gather(1, at)[:, 0], 0.0)
    s = torch.softmax(z, 1)
    hit = torch.zeros_like(s).scatter_(1, at, 1.0)
    gw = (torch.where(there, dloss.double(), 0.0) * scale)[:, None]
    # what the logits may be off by: the chain of d additions, and what the exponent's argument is rounded to
    dz = (h.double().abs() @ w.double().abs().t()).amax(1) * abs(scale) * (h.shape[1] + 3) * U
    de = 2 * dz + 4 * U * (lse.abs() + z.abs().amax(1)) * math.log2(math.e) + 130 * U
    return there, lse, loss, s, hit, gw, dz, de


def _xent_check(h, w, targets, dloss, scale, t, run):
    there, lse, loss, s, hit, gw, dz, de = _xent_ref(h, w, targets, dloss, scale)
    got_loss, got_lse, dh, dw = run()
    near(got_lse, lse, dz + de, F32)
    near(got_loss, loss, torch.where(there, 2 * dz + de + 2 * U * (lse.abs() + loss.abs()), 0.0), F32)
    p, size = (s - hit) * gw, ((s - hit).abs() * (half_step(t) * (1 + de[:, None]) + 4 * U) + s * (2 * de[:, None])) * gw.abs()
    if t == F16:
        size = size + 2.0 ** -25 * 2.0 ** -13 * gw.abs().max()          # (steps of fp16's smallest numbers under the range P is kept in)
    v, n = w.shape[0], h.shape[0]
    hh = torch.where(there[:, None], h.double(), 0.0)
    near(dh, p @ w.double(), size @ w.double().abs() + p.abs() @ w.double().abs() * (v + 40) * U, t)
    near(dw, p.t() @ hh, size.t() @ hh.abs() + p.abs().t() @ hh.abs() * (n + 8) * U, t)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("n,v,d", XENT_SHAPES)
def test_softmax_xent(t, n, v, d):
    h, w, targets, dloss = _xent_inputs(t, n, v, d, n + v + d)
    scale = 1.75

    def run(hd=h.to(DEV), wd=w.to(DEV), i=targets.to(DEV), workspace=None):
        loss, lse = embed.softmax_xent(hd, wd, i, scale=scale)
        return (loss, lse) + embed.softmax_xent_grad(hd, wd, i, lse, dloss.to(DEV), scale=scale, workspace=workspace)
    _xent_check(h, w, targets, dloss, scale, t, run)
    first = run()
    for a, b in zip(first, run(strided(h.to(DEV), 3, 1), strided(w.to(DEV), 8, 8), targets.int().to(DEV))):
        assert torch.equal(a, b)
    # a workspace that makes the smallest pieces
    least = torch.empty(_least(n, v, d, t), dtype=torch.uint8, device=DEV)
    _xent_check(h, w, targets, dloss, scale, t, lambda: run(workspace=least))


def _least(n, v, d, t):
    """The smallest workspace that the gradient takes, by asking."""
    x = torch.zeros((n, d), dtype=t, device=DEV)
    w = torch.zeros((v, d), dtype=t, device=DEV)
    f = torch.zeros(n, device=DEV)
    with pytest.raises(knn.TagoreError, match="needed") as e:
        embed.softmax_xent_grad(x, w, torch.zeros(n, dtype=torch.int64, device=DEV), f, f, workspace=torch.empty(256, dtype=torch.uint8, device=DEV))
    return int(str(e.value).split(" given, ")[1].split(" ")[0])


def test_softmax_xent_of_large_tiles():
    # tokens and rows enough for the tiles of 256, several pieces, odd ends; against fp64 on the device
    n, v, d = 2100, 30_011, 136
    for t in (BF16, F16):
        h, w, targets, dloss = _xent_inputs(t, n, v, d, 3)
        ws = torch.empty(200 << 20, dtype=torch.uint8, device=DEV)
        hd, wd, i, g = h.to(DEV), w.to(DEV), targets.to(DEV), dloss.to(DEV)
        loss, lse = embed.softmax_xent(hd, wd, i)
        one = embed.softmax_xent_grad(hd, wd, i, lse, g)
        many = embed.softmax_xent_grad(hd, wd, i, lse, g, workspace=ws[: 60 << 20])
        z = hd.double() @ wd.double().t()
        there = (i >= 0) & (i < v)
        lse64 = torch.logsumexp(z, 1)
        p = torch.softmax(z, 1)
        at = i.clamp(0, v - 1)[:, None]
        z_t = z.gather(1, at)[:, 0]
        p.scatter_add_(1, at, torch.full_like(at, -1, dtype=p.dtype))
        p *= torch.where(there, g.double(), 0.0)[:, None]
        # logits of about 10: a bound of 1e-4 on them, half a step of the type on P
        near(lse, lse64.cpu(), torch.full((n,), 1e-4), F32)
        near(loss, torch.where(there, lse64 - z_t, 0.0).cpu(), torch.full((n,), 2e-4), F32)
        for dh, dw in (one, many):
            b = half_step(t) + 4e-4
            near(dh, (p @ wd.double()).cpu(), (p.abs() @ wd.double().abs()).cpu() * b, t)
            pt = p.t().contiguous()
            near(dw, (pt @ hd.double()).cpu(), (pt.abs() @ hd.double().abs()).cpu() * b, t)


@pytest.mark.parametrize("t", [F32, BF16, F16])
def test_tokens_without_a_target_have_no_part(t):
    h, w, targets, dloss = _xent_inputs(t, 70, 300, 48, 9, ignored=False)
    keep = torch.ones(70, dtype=torch.bool)
    keep[::3] = False
    odd = h.clone()
    odd[~keep] = float("nan")
    odd[0, 5] = float("inf")
    dl = dloss.clone()
    dl[~keep] = float("nan")
    i = torch.where(keep, targets, torch.tensor([-100]))
    loss, lse = embed.softmax_xent(odd.to(DEV), w.to(DEV), i.to(DEV))
    dh, dw = embed.softmax_xent_grad(odd.to(DEV), w.to(DEV), i.to(DEV), lse, dl.to(DEV))
    l2, lse2 = embed.softmax_xent(h.to(DEV), w.to(DEV), i.to(DEV))
    dh2, dw2 = embed.softmax_xent_grad(h.to(DEV), w.to(DEV), i.to(DEV), lse2, dloss.to(DEV))
    assert torch.equal(loss, l2) and torch.equal(dh, dh2) and torch.equal(dw, dw2)
    assert (loss.cpu()[~keep] == 0).all() and (dh.cpu()[~keep] == 0).all()
    # nobody has one
    none = torch.full((70,), -1, device=DEV)
    loss, lse = embed.softmax_xent(h.to(DEV), w.to(DEV), none)
    dh, dw = embed.softmax_xent_grad(odd.to(DEV), w.to(DEV), none, lse, dl.to(DEV))
    assert (loss == 0).all() and (dh == 0).all() and (dw == 0).all()
    dh, dw = embed.softmax_xent_grad(h[:0].to(DEV), w.to(DEV), none[:0], lse[:0], lse[:0])
    assert dh.shape == (0, 48) and (dw == 0).all()


def test_softmax_xent_gradient_is_the_losses_difference():
    g = gen(11)
    h, w, targets, dloss = _xent_inputs(F32, 50, 90, 20, 11)
    loss, lse = embed.softmax_xent(h.to(DEV), w.to(DEV), targets.to(DEV), scale=0.5)
    dh, dw = embed.softmax_xent_grad(h.to(DEV), w.to(DEV), targets.to(DEV), lse, dloss.to(DEV), scale=0.5)
    wh, ww = torch.randn(h.shape, generator=g, dtype=torch.float64), torch.randn(w.shape, generator=g, dtype=torch.float64)

    def value(h, w):
        z = (h @ w.t()) * 0.5
        there = (targets >= 0) & (targets < 90)
        each = torch.logsumexp(z, 1) - z.gather(1, targets.clamp(0, 89)[:, None])[:, 0]
        return (torch.where(there, each, 0.0) * dloss.double()).sum().item()
    h, w, e = h.double(), w.double(), 1e-4
    assert abs((dh.cpu().double() * wh).sum().item() - (value(h + e * wh, w) - value(h - e * wh, w)) / (2 * e)) < 1e-4
    assert abs((dw.cpu().double() * ww).sum().item() - (value(h, w + e * ww) - value(h, w - e * ww)) / (2 * e)) < 1e-4


def test_small_weights_of_narrow_gradients():
    # fp16 keeps P in a range of its own: weights of 1e-7 do not vanish
    h, w, targets, dloss = _xent_inputs(F16, 80, 200, 64, 13)
    _, lse = embed.softmax_xent(h.to(DEV), w.to(DEV), targets.to(DEV))
    big = embed.softmax_xent_grad(h.to(DEV), w.to(DEV), targets.to(DEV), lse, dloss.to(DEV))
    small = embed.softmax_xent_grad((h.float() * 1).half().to(DEV), w.to(DEV), targets.to(DEV), lse, (dloss * 2.0 ** -10).to(DEV))
    for a, b in zip(big, small):
        # the same numbers, ten places down: what the type of the result can still show of them
        assert (a.double() * 2.0 ** -10 - b.double()).abs().max() <= 2.0 ** -25


# ---- how they are called

def test_refusals_of_the_binding():
    x = torch.zeros(4, 8, device=DEV)
    i = torch.zeros(4, dtype=torch.int64, device=DEV)
    w = torch.zeros(8, device=DEV)
    q, s = embed.quantize_rows(x)
    for call in (lambda: embed.lookup(x.t(), i), lambda: embed.lookup(x, i.float()), lambda: embed.lookup(x.double(), i), lambda: embed.lookup(x[0], i),
                 lambda: embed.lookup(x[:1].expand(4, 8), i), lambda: embed.lookup_grad(x[:3], i, 5), lambda: embed.lookup_grad(x, i, 5, out=x),
                 lambda: embed.lookup_grad(x, i, 4, out=x.half()), lambda: embed.add_rms_norm(x, w[:7]), lambda: embed.add_rms_norm(x, w.half()),
                 lambda: embed.add_rms_norm(x, w, residual=x[:3]), lambda: embed.add_rms_norm(x, w, residual=x.half()),
                 lambda: embed.add_rms_norm_grad(x, x, w, s.half()), lambda: embed.matmul_q8(q, s, q[:, :4].contiguous(), s),
                 lambda: embed.matmul_q8(q, s[:3], q, s), lambda: embed.matmul_q8(q[:, :4], s, q[:, :4], s), lambda: embed.matmul_q8(q, s, q, s, bias=w),
                 lambda: embed.matmul_q8(q, s, q, s, out_dtype=torch.float64), lambda: embed.softmax_xent(x, x.half(), i), lambda: embed.softmax_xent(x, x, i[:3]),
                 lambda: embed.softmax_xent(x, x[:, :4], i), lambda: embed.softmax_xent_grad(x, x, i, s, s[:2]), lambda: embed.dequantize_rows(q, s, torch.int8)):
        with pytest.raises((TypeError, ValueError)):
            call()
    with pytest.raises(knn.TagoreError, match="outside 1..8192"):
        embed.add_rms_norm(torch.zeros(2, 8193, device=DEV), torch.zeros(8193, device=DEV))
    with pytest.raises(knn.TagoreError, match="eps"):
        embed.add_rms_norm(x, w, eps=-1.0)
    for f in (lambda z: embed.lookup(x, i[:0]), lambda z: embed.add_rms_norm(z, w)[0], lambda z: embed.quantize_rows(z)[0],
              lambda z: embed.matmul_q8(q[:0], s[:0], q, s), lambda z: embed.softmax_xent(z, x, i[:0])[0]):
        assert f(x[:0]).shape[0] == 0


def _step(table, ids, weight, targets, dloss):
    x = embed.lookup(table, ids, scale=2.0)
    y, r, rstd = embed.add_rms_norm(x, weight, residual=x)
    loss, lse = embed.softmax_xent(y, table, targets)
    dy, dtable = embed.softmax_xent_grad(y, table, targets, lse, dloss)
    dx, dweight = embed.add_rms_norm_grad(dy, r, weight, rstd)
    embed.lookup_grad(dx, ids, table.shape[0], scale=4.0, out=dtable)
    q, s, _ = embed.add_rms_norm_q8(x, weight, residual=x)
    tq, ts = embed.quantize_rows(table)
    return loss, dtable, dweight, embed.matmul_q8(q, s, tq, ts)


def _step_inputs(seed, n, v, d, t=BF16):
    g = gen(seed)
    return (torch.randn(v, d, generator=g).to(t).to(DEV), torch.randint(0, v, (n,), generator=g).to(DEV), (1 + 0.1 * torch.randn(d, generator=g)).to(t).to(DEV),
            torch.randint(-1, v, (n,), generator=g).to(DEV), (torch.rand(n, generator=g) / n).to(DEV))


@pytest.mark.parametrize("n", [48, 20_000])
def test_a_step_in_a_graph(n):
    state = [x.clone() for x in _step_inputs(0, n, 1500, 64)]
    _step(*state)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _step(*state)
    for seed in range(4):
        for a, b in zip(state, _step_inputs(seed, n, 1500, 64)):
            a.copy_(b)
        want = [x.clone() for x in _step(*state)]
        for o in out:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b)


def test_on_another_stream():
    inputs = _step_inputs(4, 300, 700, 96, F32)
    want = _step(*inputs)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        big = torch.randn(4096, 4096, device=DEV)
        for _ in range(20):
            big = big @ big * 1e-3                   # the stream is busy: a call on another one would be in front
        late = [x.clone() for x in inputs]
        got = _step(*late)
    side.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)
