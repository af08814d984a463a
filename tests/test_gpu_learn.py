"""The operators of include/tagore_learn.h against plain forms in 64 bits.

Tolerances are bounds, from the roundings that a result goes through: half a step of its type, and for every fp32 sum its longest chain
of additions times 2^-24 of the sum of the terms' magnitudes.
"""
import math

import pytest
import torch

from paper_2508_08744_amd import embed, knn, learn

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
    flat = torch.full((offset + n * (d + extra),), float("nan"), dtype=x.dtype, device=x.device)
    y = flat[offset:].view(n, d + extra)[:, :d]
    y.copy_(x)
    return y


def inputs(t, n, v, d, seed, ignored=True):
    g = gen(seed)
    w = (torch.randn(v, d, generator=g) / math.sqrt(d)).to(t)
    targets = torch.randint(0, v, (n,), generator=g)
    h = (torch.randn(n, d, generator=g) + 3 * w[targets].float()).to(t)
    if ignored and n > 2:
        targets[::7] = -1
        targets[3::31] = v
    return h, w, targets


class Ref:
    """Everything in 64 bits, and what the fp32 logits and exponents may be off by."""

    def __init__(self, h, w, targets, scale):
        v, d = w.shape
        self.h, self.w, self.scale = h, w, scale
        self.there = (targets >= 0) & (targets < v)
        self.at = targets.clamp(0, v - 1)[:, None]
        self.z = (h.double() @ w.double().t()) * scale
        self.lse = torch.logsumexp(self.z, 1)
        self.logp = torch.where(self.there, self.z.gather(1, self.at)[:, 0] - self.lse, 0.0)
        self.log_p = self.z - self.lse[:, None]
        self.p = self.log_p.exp()
        self.entropy = -(self.p * self.log_p).sum(1)
        # the chain of d additions and the factor's product; what an exponent's argument is rounded to, and the chains of its sum
        self.dz = (h.double().abs() @ w.double().abs().t()).amax(1) * abs(scale) * (d + 3) * U
        self.de = 2 * self.dz + 4 * U * (self.lse.abs() + self.z.abs().amax(1)) * math.log2(math.e) + 130 * U
        self.dlse = self.dz + self.de
        # H changes by sum p |log p + H| <= 2 H times a relative change of p; the sums of 2^t and t 2^t have chains of their own
        self.dentropy = (2 * self.entropy + 1) * (self.dz + self.de) + 300 * U * (1 + math.log(v))

    def check(self, logp, entropy, lse):
        near(lse, self.lse, self.dlse, F32)
        near(entropy, self.entropy, self.dentropy, F32)
        near(logp, self.logp, torch.where(self.there, 2 * self.dz + self.de + 2 * U * (self.lse.abs() + self.logp.abs()), 0.0), F32)

    def check_best(self, rows, row_logp, top):
        n, v = self.z.shape
        k = min(top, v)
        z, at = torch.sort(self.z, dim=1, descending=True, stable=True)       # (equal ones by the lower row)
        assert torch.equal(rows.cpu()[:, :k].long(), at[:, :k])
        near(row_logp[:, :k], z[:, :k] - self.lse[:, None], (self.dlse + 2 * U * self.lse.abs())[:, None], F32)
        assert (rows[:, k:] == -1).all() and (row_logp[:, k:] == -math.inf).all()


SHAPES = [(1, 1, 1, 1), (2, 3, 8, 5), (1, 700, 64, 8), (30, 129, 96, 32), (33, 1000, 50, 20), (64, 257, 128, 1), (65, 300, 40, 7), (130, 515, 33, 32), (300, 2100, 72, 3),
          (257, 8000, 130, 8), (1, 20_001, 16, 32), (31, 9000, 24, 5), (50, 20_000, 40, 9),
          (23, 553, 91, 20), (14, 1116, 56, 28), (3000, 300, 24, 32), (3000, 1000, 16, 32), (7, 33, 8, 32)]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("n,v,d,top", SHAPES)
def test_log_probs(t, n, v, d, top):
    h, w, targets = inputs(t, n, v, d, n + v + d)
    scale = 1.75
    ref = Ref(h, w, targets, scale)
    hd, wd, i = h.to(DEV), w.to(DEV), targets.to(DEV)
    first = learn.log_probs(hd, wd, i, scale=scale, top=top)
    ref.check(*first[:3])
    ref.check_best(*first[3:], top)
    # other distances and starts of the rows, narrow targets: the same bits
    for a, b in zip(first, learn.log_probs(strided(hd, 3, 1), strided(wd, 8, 8), i.int(), scale=scale, top=top)):
        assert torch.equal(a, b)
    for a, b in zip(first, learn.log_probs(strided(hd, 8, 8), strided(wd, 5, 3), i, scale=scale, top=top)):
        assert torch.equal(a, b)
    # of one kind of tiles nothing depends on what else is asked for
    logp, entropy, lse, rows, row_logp = learn.log_probs(hd, wd, scale=scale, top=top)
    assert logp is None and all(torch.equal(a, b) for a, b in zip((entropy, lse, rows, row_logp), first[1:]))
    none = learn.log_probs(hd, wd, i, scale=scale)
    assert all(torch.equal(a, b) for a, b in zip(none[:3], first[:3])) and none[3].shape == none[4].shape == (n, 0)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("n", [1, 40, 100, 300, 3000])
def test_of_negative_and_no_scale(t, n):
    h, w, targets = inputs(t, n, 900, 48, n)
    hd, wd, i = h.to(DEV), w.to(DEV), targets.to(DEV)
    for scale in (-0.75, 0.0):
        ref = Ref(h, w, targets, scale)
        got = learn.log_probs(hd, wd, i, scale=scale, top=6)
        ref.check(*got[:3])
        ref.check_best(*got[3:], 6)


def _log_probs_at_the_boundary(h, w, top, targets=None, targets64=1, logp=None):
    """tg_log_probs itself: (rc, logp, entropy, lse, rows, row_logp)."""
    L, t = learn.lib(), embed.DTYPES[h.dtype]
    (n, d), v = h.shape, w.shape[0]
    entropy, lse = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    rows, row_logp = torch.empty(n, top, dtype=torch.int32, device=DEV), torch.empty(n, top, device=DEV)
    nbytes = L.tg_log_probs_workspace(n, v, d, t, top, 0)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=DEV)
    rc = L.tg_log_probs(h.data_ptr(), d, w.data_ptr(), d, t, n, v, d, embed._ptr(targets), targets64, 1.0, top, embed._ptr(logp), entropy.data_ptr(), lse.data_ptr(),
                        rows.data_ptr(), row_logp.data_ptr(), ws.data_ptr(), nbytes, embed._stream())
    return rc, logp, entropy, lse, rows, row_logp


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("n,v", [(1, 700), (40, 3000), (256, 900), (257, 900), (3000, 900), (450, 30_000)])
def test_without_targets_every_log_probability_is_0(t, n, v):
    """At the C boundary the targets may be missing where their log probabilities are asked for: no token has one."""
    h, w, _ = inputs(t, n, v, 24, n)
    hd, wd = h.to(DEV), w.to(DEV)
    for top in (0, 5):
        want = learn.log_probs(hd, wd, top=top)
        for targets64 in (0, 1):
            got = _log_probs_at_the_boundary(hd, wd, top, targets64=targets64, logp=torch.full((n,), 7.0, device=DEV))
            assert got[0] == 0 and (got[1] == 0).all()
            for a, b in zip(got[2:], want[1:]):
                assert torch.equal(a, b)


def _device_ref(hd, wd, scale, top, step=4096):
    """lse, entropy and the best rows in 64 bits, on the device, some tokens at a time."""
    out = []
    w64 = wd.double().t().contiguous()
    for a in hd.split(step):
        z = (a.double() @ w64) * scale
        lse = torch.logsumexp(z, 1)
        log_p = z - lse[:, None]
        out.append((lse, -(log_p.exp() * log_p).sum(1)) + tuple(torch.topk(z, top, dim=1)))
    return [torch.cat(x) for x in zip(*out)]


@pytest.mark.parametrize("t,n,v,d,top", [(BF16, 2100, 30_011, 136, 8), (F16, 2100, 30_011, 136, 32), (F32, 900, 30_011, 40, 20), (BF16, 400, 6000, 64, 5),
                                         (BF16, 70_000, 40_000, 8, 2), (BF16, 2, 1_000_003, 64, 10), (F16, 60, 300_000, 64, 31), (F32, 17, 100_000, 200, 16),
                                         (BF16, 8192, 2000, 64, 32), (BF16, 8192, 9000, 64, 32), (F16, 3000, 1100, 64, 32), (BF16, 100, 1_000_003, 24, 32), (F16, 600, 3_000_001, 16, 6), (F32, 70, 20_000_003, 12, 4)])
def test_log_probs_of_many_tiles(t, n, v, d, top):
    g = gen(n)
    w = (torch.randn(v, d, generator=g) / math.sqrt(d)).to(t).to(DEV)
    h = (2 * torch.randn(n, d, generator=g)).to(t).to(DEV)
    targets = torch.randint(-1, v, (n,), generator=g).to(DEV)
    logp, entropy, lse, rows, row_logp = learn.log_probs(h, w, targets, top=top)
    lse64, entropy64, z, at = _device_ref(h, w, 1.0, top)
    # logits up to about 12, their sums of magnitudes up to 60: (d + 3) U of these, and the exponents' part
    dz = 60 * (d + 3) * U
    dlse = torch.full((n,), 3 * dz + (4 * 30 * 1.5 + 130) * U)
    near(lse, lse64.cpu(), dlse, F32)
    near(entropy, entropy64.cpu(), (2 * entropy64.cpu() + 1) * dlse + 300 * U * (1 + math.log(v)), F32)
    assert torch.equal(rows.long(), at)
    near(row_logp, (z - lse64[:, None]).cpu(), dlse[:, None] + 60 * U, F32)
    there = targets >= 0
    mine = (h.double() * w[targets.clamp_min(0)].double()).sum(1)
    near(logp, torch.where(there, mine - lse64, 0.0).cpu(), dlse + dz + 60 * U, F32)
    assert (logp[~there] == 0).all()


@pytest.mark.parametrize("n", [2, 11])
def test_a_table_past_32_bits_of_elements(n):
    """2^29 rows and some, of zeros but for a few far apart."""
    v, d = (1 << 29) + 1001, 8
    w = torch.zeros(v, d, dtype=BF16, device=DEV)
    at = torch.tensor([3, (1 << 28) + 5, (1 << 29) - 1, (1 << 29) + 7, v - 1], device=DEV)
    w[at] = torch.tensor([[12.0], [14.0], [11.0], [13.0], [10.0]], device=DEV).to(BF16).expand(5, d)
    h = torch.full((n, d), 0.25, dtype=BF16, device=DEV)
    h[1] = -0.25
    targets = torch.full((n,), v - 1, device=DEV)
    logp, entropy, lse, rows, row_logp = [x.cpu() for x in learn.log_probs(h, w, targets, top=4)]
    for y, sign in ((0, 1.0), (1, -1.0), (n - 1, 1.0 if n > 2 else -1.0)):
        z = sign * torch.tensor([24.0, 28.0, 22.0, 26.0, 20.0], dtype=torch.float64)
        total = math.log(v - 5 + z.exp().sum().item())
        p = (z - total).exp()
        h64 = -(p * (z - total)).sum().item() + (v - 5) * math.exp(-total) * total
        # every part of the table is joined once: a chain of 64 within a tile and some 100 over the parts
        bound = 400 * U * (1 + total)
        assert abs(lse[y].item() - total) <= bound and abs(entropy[y].item() - h64) <= 30 * bound
        assert abs(logp[y].item() - (z[4].item() - total)) <= bound + 40 * U
        if sign > 0:
            assert rows[y].tolist() == [(1 << 28) + 5, (1 << 29) + 7, 3, (1 << 29) - 1]
            assert ((row_logp[y].double() - (torch.tensor([28.0, 26.0, 24.0, 22.0]) - total)).abs() <= bound + 40 * U).all()


# ---- order of the best rows

@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("n,v", [(1, 700), (9, 5000), (40, 5000), (100, 3000), (300, 2000), (300, 20_000), (3000, 4000), (700, 20_000)])
def test_equal_logits_go_to_the_lower_row(t, n, v):
    # small whole numbers: logits are exact, and most of them equal to others; some tokens' are all 0, the table's rows come several times
    g = gen(n + v)
    w = torch.randint(-2, 3, (v, 12), generator=g).float()
    w[v // 2:] = w[: v - v // 2]
    h = torch.randint(-2, 3, (n, 12), generator=g).float()
    h[::5] = 0
    z = h.double() @ w.double().t()
    best, at = torch.sort(z, dim=1, descending=True, stable=True)
    lse = torch.logsumexp(z, 1)
    for top in (1, 7, 32):
        _, _, _, rows, row_logp = learn.log_probs(h.to(t).to(DEV), w.to(t).to(DEV), top=top)
        assert torch.equal(rows.cpu().long(), at[:, :top])
        near(row_logp, best[:, :top] - lse[:, None], torch.full((n, 1), 400 * U * 12), F32)
    # one row, v times
    same = w[:1].expand(v, 12).contiguous()
    _, _, _, rows, _ = learn.log_probs(h[:64].to(t).to(DEV), same.to(t).to(DEV), top=20)
    assert torch.equal(rows.cpu(), torch.arange(20, dtype=torch.int32).expand(min(n, 64), 20))


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("n,v,d", [(1, 3000, 64), (20, 5000, 256), (100, 3000, 96), (300, 3000, 512), (300, 30_000, 128), (450, 30_000, 96)])
def test_order_below_the_roundings_of_the_logits(t, n, v, d):
    """Large terms that cancel leave logits which 32 bits have no place of: their order is that of the exact sums."""
    g = gen(d)
    w = torch.randn(v, d, generator=g)
    big = 2.0 ** 12 * torch.randn(v, d // 4, generator=g)
    w[:, : d // 4] = big
    w[:, d // 2: d // 2 + d // 4] = -big.to(t).float()
    w = w.to(t)
    h = torch.randn(n, d, generator=g)
    h[:, : d // 4] = 1.0
    h[:, d // 2: d // 2 + d // 4] = 1.0
    h = h.to(t)
    scale = 2.0 ** -4
    # (what the large terms leave: nothing; the logits are small numbers, and the tiles' are off by more than most differ)
    z = (h.double() @ w.double().t()) * scale
    assert z.abs().max() < 40
    best, at = torch.sort(z, dim=1, descending=True, stable=True)
    _, _, _, rows, _ = learn.log_probs(h.to(DEV), w.to(DEV), scale=scale, top=10)
    assert torch.equal(rows.cpu().long(), at[:, :10])


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("n,v,d,longer", [(1, 3000, 1024, 1000), (20, 5000, 2048, 400), (40, 9000, 512, 4000), (100, 3000, 1024, 1000), (300, 3000, 2048, 400), (450, 30_000, 512, 3000)])
def test_order_beside_a_row_far_longer_than_the_others(t, n, v, d, longer):
    """What a logit may be off by goes by the longest row of the table: thousands of rows are then not out of reach of the best ones, and are scored in 64 bits."""
    g = gen(n + d)
    w = torch.randn(v, d, generator=g) / math.sqrt(d)
    long = v // 3
    w[long] *= longer
    w = w.to(t)
    h = (2 * torch.randn(n, d, generator=g)).to(t)
    h[-1] = -h[0]                                              # (the long row is first for one of them, or last)
    z = h.double() @ w.double().t()
    best, at = torch.sort(z, dim=1, descending=True, stable=True)
    # the bound of d products and sums at a step each, twice: more rows than a list of 1024 holds
    reach = 2 * (d + 2) * 2.0 ** -23 * h.double().norm(dim=1) * w.double().norm(dim=1).max()
    assert (z >= (best[:, 7] - reach)[:, None]).sum(1).min() > 1024
    _, _, _, rows, row_logp = learn.log_probs(h.to(DEV), w.to(DEV), top=8)
    assert torch.equal(rows.cpu().long(), at[:, :8])
    lse = torch.logsumexp(z, 1)
    # logits that count are the long row's, up to its own bound, or below 16, and the exponents' part
    size = z.abs().amax(1)
    dz = (h.double().abs() @ w.double().abs().t()).amax(1) * (d + 3) * U
    near(row_logp, best[:, :8] - lse[:, None], (3 * dz + 8 * U * (lse.abs() + size) + 130 * U)[:, None] + 2 * U * (best[:, :8] - lse[:, None]).abs(), F32)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("n,v,d", [(1, 3000, 1024), (20, 5000, 1024), (40, 9000, 512), (100, 3000, 1024), (300, 3000, 512), (450, 30_000, 512), (3000, 2000, 256)])
@pytest.mark.parametrize("each", [50, 1000])
def test_order_where_many_tiles_have_a_long_row(t, n, v, d, each):
    """Rows far longer than the others along what no token has: ordinary logits, and nothing of their tiles' out of reach of the best ones, more than a list holds."""
    g = gen(n + v)
    w = torch.randn(v, d, generator=g) / math.sqrt(d)
    w[::each, 0] = 20_000.0
    w = w.to(t)
    h = 2 * torch.randn(n, d, generator=g)
    h[:, 0] = 0
    h = h.to(t)
    z = h.double() @ w.double().t()
    best, at = torch.sort(z, dim=1, descending=True, stable=True)
    # a long row's part in its tile's bound, of d products and sums at a step each, on either side
    reach = 2 * (d + 2) * 2.0 ** -23 * h.double().norm(dim=1) * 20_000
    assert each > 50 or (z >= (best[:, 7] - reach)[:, None]).sum(1).min() > 1024
    _, _, _, rows, _ = learn.log_probs(h.to(DEV), w.to(DEV), top=8)
    assert torch.equal(rows.cpu().long(), at[:, :8])


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("n,v,d", [(1, 700, 64), (1, 30_000, 64), (20, 5000, 256), (40, 9000, 128), (100, 3000, 96), (300, 3000, 512), (300, 30_000, 128), (450, 30_000, 96), (3000, 1000, 64)])
@pytest.mark.parametrize("where", ["together", "apart"])
def test_order_where_some_rows_logits_are_what_large_terms_leave(t, n, v, d, where):
    """Some rows' logits are off by more than the others are apart, those in tiles of ordinary rows beside them are not: each is looked at as its own tile asks for."""
    g = gen(n + v + d)
    w = 4 * torch.randn(v, d, generator=g) / math.sqrt(d)
    at = torch.arange(v // 3, v // 3 + 50) if where == "together" else torch.randperm(v, generator=g)[:12]
    big = 2.0 ** 12 * torch.randn(len(at), d // 4, generator=g)
    w[at, : d // 4] = big
    w[at, d // 2: d // 2 + d // 4] = -big.to(t).float()
    w = w.to(t)
    h = torch.randn(n, d, generator=g)
    h[:, : d // 4] = 1.0
    h[:, d // 2: d // 2 + d // 4] = 1.0
    h = h.to(t)
    z = h.double() @ w.double().t()
    assert z.abs().max() < 60
    best, order = torch.sort(z, dim=1, descending=True, stable=True)
    for top in (1, 10, 32):
        _, _, _, rows, _ = learn.log_probs(h.to(DEV), w.to(DEV), top=top)
        assert torch.equal(rows.cpu().long(), order[:, :top])


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("n,v", [(1, 3000), (50, 3000), (100, 3000), (450, 30_000)])
def test_order_of_rows_of_the_smallest_numbers(t, n, v):
    """Values below the type's normal ones: whatever the tiles make of them, the best rows are those of the exact sums."""
    g = gen(n)
    tiny = torch.finfo(t).tiny
    w = (torch.randint(-100, 101, (v, 24), generator=g).double() * tiny / 128).to(t)
    h = torch.randn(n, 24, generator=g).to(t)
    scale = float(torch.tensor(0.03 / tiny).float()) if t == F16 else 2.0 ** 124
    z = (h.double() @ w.double().t()) * scale
    _, _, _, rows, _ = learn.log_probs(h.to(DEV), w.to(DEV), scale=scale, top=12)
    assert torch.equal(rows.cpu().long(), torch.sort(z, dim=1, descending=True, stable=True)[1][:, :12])


@pytest.mark.parametrize("t", [F32, BF16])
@pytest.mark.parametrize("n,v", [(1, 3000), (50, 3000), (100, 3000), (300, 2100), (450, 30_000)])
@pytest.mark.parametrize("size", [-58, -63, -65, -68])
def test_order_of_products_of_the_smallest_size(t, n, v, size):
    """Values that are normal numbers, whose products are not, brought up by the factor: whatever is left of the sums, the best rows are those of the exact ones."""
    g = gen(n)
    w = (torch.randn(v, 24, generator=g) * 2.0 ** size).to(t)
    h = (torch.randn(n, 24, generator=g) * 2.0 ** size).to(t)
    scale = 2.0 ** 126
    z = (h.double() @ w.double().t()) * scale
    _, _, _, rows, _ = learn.log_probs(h.to(DEV), w.to(DEV), scale=scale, top=12)
    assert torch.equal(rows.cpu().long(), torch.sort(z, dim=1, descending=True, stable=True)[1][:, :12])


# ---- infinite and undefined logits

@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("n,v", [(3, 40), (40, 3000), (100, 2100), (300, 2100), (300, 30_000), (450, 30_000)])
def test_infinite_logits(t, n, v):
    w = torch.full((v, 8), 2.0 ** -10)
    w[v // 2, 3] = -2.0
    w[v // 3, 3] = 0.5
    h = torch.zeros(n, 8)
    h[:, 3] = 1.0
    h[1, 3] = math.inf                                  # +inf everywhere but at one row
    h[2, 3] = -math.inf                                 # -inf everywhere but at one row
    targets = torch.full((n,), v // 2)
    w_t = w.to(t)
    col = w_t[:, 3].double()
    got = [x.cpu() for x in learn.log_probs(h.to(t).to(DEV), w_t.to(DEV), targets.to(DEV), top=4)]
    logp, entropy, lse, rows, row_logp = got
    # an ordinary token beside them is as without them
    z = col
    want = torch.logsumexp(z, 0)
    p = torch.softmax(z, 0)
    at = [0] + list(range(3, n))
    assert ((lse[at].double() - want).abs() <= 200 * U + 4 * U * want).all()
    assert ((entropy[at].double() + (p * torch.log_softmax(z, 0)).sum()).abs() <= 1200 * U * math.log(v)).all()
    order = torch.sort(z, descending=True, stable=True)[1][:4]
    assert (rows[at].long() == order).all()
    # h is 0 in the other columns and infinite in one: the products there are exact infinities
    assert lse[1] == math.inf and entropy[1].isnan() and logp[1] == -math.inf
    first = [v_ for v_ in range(v) if v_ != v // 2][:4]
    assert rows[1].tolist() == first and row_logp[1].isnan().all()
    assert lse[2] == math.inf and entropy[2].isnan() and logp[2].isnan()
    assert rows[2].tolist() == [v // 2] + first[:3] and row_logp[2, 0].isnan() and (row_logp[2, 1:] == -math.inf).all()
    # all of a token's logits are -infinity: nothing is defined but their order
    low = torch.ones(v, 8)
    h = torch.zeros(n, 8)
    h[0] = -math.inf
    logp, entropy, lse, rows, row_logp = [x.cpu() for x in learn.log_probs(h.to(t).to(DEV), low.to(t).to(DEV), targets.to(DEV), top=4)]
    assert lse[0] == -math.inf and entropy[0].isnan() and logp[0].isnan() and rows[0].tolist() == [0, 1, 2, 3]
    assert ((lse[1:] - math.log(v)).abs() < 1e-5).all()
    # a few are: they have no part in the entropy
    some = torch.zeros(v, 8)
    some[::3, 0] = -math.inf
    h = torch.ones(n, 8)
    logp, entropy, lse, rows, row_logp = [x.cpu() for x in learn.log_probs(h.to(t).to(DEV), some.to(t).to(DEV), torch.zeros(n, dtype=torch.int64, device=DEV), top=4)]
    count = v - (v + 2) // 3
    assert (logp == -math.inf).all() and ((lse - math.log(count)).abs() < 1e-5).all() and ((entropy - math.log(count)).abs() < 1e-5).all()
    assert (rows == torch.tensor([1, 2, 4, 5])).all()


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("n,v", [(3, 40), (40, 3000), (100, 2100), (300, 2100), (300, 30_000), (2500, 2000), (450, 30_000)])
def test_a_nan_stays_with_its_token(t, n, v):
    h, w, targets = inputs(t, n, v, 24, 5)
    want = learn.log_probs(h.to(DEV), w.to(DEV), targets.to(DEV), top=5)
    odd = h.clone()
    odd[1, 3] = math.nan
    got = learn.log_probs(odd.to(DEV), w.to(DEV), targets.to(DEV), top=5)
    keep = [0] + list(range(2, n))
    for a, b in zip(got, want):
        assert torch.equal(a[keep], b[keep])
    logp, entropy, lse, rows, row_logp = (x[1] for x in got)
    assert entropy.isnan() and lse.isnan() and (rows == -1).all() and row_logp.isnan().all()
    assert logp.isnan() if 0 <= targets[1] < v else logp == 0
    # one in the table is everyone's
    odd = w.clone()
    odd[v - 1, 7] = math.nan
    logp, entropy, lse, rows, row_logp = learn.log_probs(h.to(DEV), odd.to(DEV), targets.to(DEV), top=5)
    assert entropy.isnan().all() and lse.isnan().all() and (rows == -1).all() and row_logp.isnan().all()


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("n,v", [(3, 40), (40, 3000), (100, 2100), (300, 30_000), (450, 30_000)])
def test_huge_logits(t, n, v):
    """One column of h and w makes the logits, exact products of a size whose exponents leave fp32 by far: one row has the whole softmax, or logits are infinite."""
    g = gen(n)
    w = torch.zeros(v, 8)
    w[:, 3] = torch.rand(v, generator=g) * 2.0 ** -10
    w[v // 2, 3] = 1.5
    w = w.to(t)
    h = torch.zeros(n, 8)
    h[:, 3] = 1.0
    h[n // 2:, 3] = -1.0
    targets = torch.randint(0, v, (n,), generator=g)
    targets[1] = v // 2
    for scale in (1e6, 3e9, 1e12, 1e30, 2e38, -1e30, 3e38):
        z = (h[:, 3:4].double() @ w[:, 3:4].double().t()) * torch.tensor(scale).double()
        logp, entropy, lse, rows, row_logp = [x.cpu() for x in learn.log_probs(h.to(t).to(DEV), w.to(DEV), targets.to(DEV), scale=scale, top=5)]
        best, at = torch.sort(z, dim=1, descending=True, stable=True)
        assert torch.equal(rows.long(), at[:, :5])
        finite = z.amax(1) < 3.4e38
        assert (lse[~finite] == math.inf).all() and entropy[~finite].isnan().all()
        lse64 = torch.logsumexp(z, 1)
        assert ((lse.double() - lse64).abs() <= 4 * U * lse64.abs() + 200 * U * math.log(v))[finite].all()
        p = torch.softmax(z, 1)
        h64 = -torch.where(p > 0, p * torch.log_softmax(z, 1), 0.0).sum(1)
        # an exponent's difference is rounded at the size of the logits, and log p and p with it where others count at all
        size = torch.where(h64 > 1e-30, z.abs().amax(1), 0.0)
        assert ((entropy.double() - h64).abs() <= (2 * h64 + 1) * 8 * U * size + 300 * U * (1 + math.log(v)))[finite].all()
        want = (z.gather(1, targets[:, None])[:, 0] - lse64).float().double()           # (what fp32 does not hold is infinite)
        fine = finite & torch.isfinite(want)
        assert ((logp.double() - want).abs() <= 8 * U * (lse64.abs() + want.abs()) + 200 * U * math.log(v))[fine].all()
        assert (row_logp <= 0).logical_or(row_logp.isnan())[finite].all()


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("n,v", [(4, 40), (256, 700), (300, 3000), (450, 30_000)])
def test_no_log_probability_is_above_0(t, n, v):
    """The target has all of the mass that fp32 sees: exponents of the largest logit are rounded at its size, some of them down."""
    g = gen(v)
    w = torch.zeros(v, 8)
    w[v // 2, 3] = 1.0
    h = torch.zeros(n, 8)
    h[:, 3] = torch.exp(math.log(50) + torch.rand(n, generator=g) * math.log(1000))
    h = h.to(t)
    targets = torch.full((n,), v // 2)
    targets[::9] = 0
    for scale in (1.0, 1.1):
        logp, _, lse, rows, row_logp = [x.cpu() for x in learn.log_probs(h.to(DEV), w.to(t).to(DEV), targets.to(DEV), scale=scale, top=3)]
        assert (logp <= 0).all() and (row_logp <= 0).all() and (rows[:, 0] == v // 2).all()
        # z = scale h (one product), the others are 0: lse is z and less than v e^-50
        z = h[:, 3].double() * torch.tensor(scale, dtype=F32).double()
        assert ((lse.double() - z).abs() <= (4 * z + 200 * math.log(v)) * U).all()
        want = torch.where(targets == 0, -z, 0.0)
        assert ((logp.double() - want).abs() <= (8 * z + 200 * math.log(v)) * U).all()


@pytest.mark.parametrize("t", [F32, BF16])
def test_logits_beyond_fp32(t):
    """Sums that fp32 does not hold: lse is infinite, and the best rows are those of the exact sums."""
    g = gen(2)
    w = torch.randn(500, 8, generator=g).to(t)
    h = torch.full((3, 8), 3e38).to(t)
    z = h.double() @ w.double().t()
    _, entropy, lse, rows, _ = learn.log_probs(h.to(DEV), w.to(DEV), top=6)
    fine = ~torch.isnan(lse).cpu()                      # (inf - inf within a sum is a NaN, and then there are no best rows)
    assert (~torch.isfinite(lse)).all() and entropy.isnan().all()
    assert torch.equal(rows.cpu()[fine].long(), torch.sort(z, dim=1, descending=True, stable=True)[1][fine, :6])
    assert (rows.cpu()[~fine] == -1).all()


# ---- gradients

def _grad_ref(ref, dlogp, dentropy):
    s = ref.scale
    a = torch.where(ref.there, dlogp.double(), 0.0)[:, None]
    b = dentropy.double()[:, None] if dentropy is not None else torch.zeros_like(a)
    hit = torch.zeros_like(ref.p).scatter_(1, ref.at, 1.0)
    inner = a + b * (ref.log_p + ref.entropy[:, None])
    return s * (a * hit - ref.p * inner), hit, a, b, inner


def _grad_check(ref, dlogp, dentropy, t, dh, dw):
    s = abs(ref.scale)
    p, hit, a, b, inner = _grad_ref(ref, dlogp, dentropy)
    part = (ref.there | (b[:, 0] != 0))[:, None]
    de = ref.de[:, None]
    # P: half a step of the type, p's relative error, what log p + H is off by beside it, and a few roundings of its parts
    parts = a.abs() * hit + ref.p * (a.abs() + b.abs() * (ref.log_p.abs() + ref.entropy[:, None]))
    size = s * (p.abs() / s * half_step(t) * (1 + de) + ref.p * inner.abs() * 2 * de + ref.p * b.abs() * (2 * de + 2 * ref.dentropy[:, None]) + parts * 8 * U)
    if t == F16:
        # (steps of fp16's smallest numbers under the range P is kept in)
        most = s * (a.abs() + b.abs() * (ref.entropy[:, None] + 0.375)).max()
        size = size + 2.0 ** -25 * 2.0 ** -13 * most
    v, n = ref.w.shape[0], ref.h.shape[0]
    hh = torch.where(part, ref.h.double(), 0.0)
    w = ref.w.double()
    near(dh, p @ w, size @ w.abs() + p.abs() @ w.abs() * (v + 40) * U, t)
    if dw is not None:
        near(dw, p.t() @ hh, size.t() @ hh.abs() + p.abs().t() @ hh.abs() * (n + 8) * U, t)


def _least(n, v, d, t, table):
    """The smallest workspace that the gradient takes, by asking."""
    x, w, f = torch.zeros((n, d), dtype=t, device=DEV), torch.zeros((v, d), dtype=t, device=DEV), torch.zeros(n, device=DEV)
    with pytest.raises(knn.TagoreError, match="needed") as e:
        learn.log_probs_grad(x, w, torch.zeros(n, dtype=torch.int64, device=DEV), f, f, table=table, workspace=torch.empty(256, dtype=torch.uint8, device=DEV))
    return torch.empty(int(str(e.value).split(" given, ")[1].split(" ")[0]), dtype=torch.uint8, device=DEV)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("n,v,d", [s[:3] for s in SHAPES])
def test_gradients(t, n, v, d):
    h, w, targets = inputs(t, n, v, d, n + v + d)
    ref = Ref(h, w, targets, 1.75)
    g = gen(7)
    dlogp, dentropy = torch.randn(n, generator=g), 0.3 * torch.randn(n, generator=g)
    dentropy[1::4] = 0
    hd, wd, i, a, b = (x.to(DEV) for x in (h, w, targets, dlogp, dentropy))
    logp, entropy, lse, _, _ = learn.log_probs(hd, wd, i, scale=1.75)

    def run(hd=hd, wd=wd, i=i, **more):
        return learn.log_probs_grad(hd, wd, i, lse, a, entropy, b, scale=1.75, **more)
    first = run()
    _grad_check(ref, dlogp, dentropy, t, *first)
    for x, y in zip(first, run(strided(hd, 3, 1), strided(wd, 8, 8), i.int())):
        assert torch.equal(x, y)
    _grad_check(ref, dlogp, dentropy, t, *run(workspace=_least(n, v, d, t, True)))
    # the table stays as it is
    dh, dw = run(table=False)
    assert dw is None
    _grad_check(ref, dlogp, dentropy, t, dh, None)
    dh, dw = run(table=False, workspace=_least(n, v, d, t, False))
    _grad_check(ref, dlogp, dentropy, t, dh, None)
    # without the entropy it is the cross entropy's gradient, bit for bit
    got = learn.log_probs_grad(hd, wd, i, lse, a, scale=1.75)
    _grad_check(ref, dlogp, None, t, *got)
    for x, y in zip(got, embed.softmax_xent_grad(hd, wd, i, lse, -a, scale=1.75)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("t", [BF16, F16])
def test_gradients_of_large_tiles(t):
    # tokens and rows enough for the tiles of 256, one piece and several, odd ends; against fp64 on the device
    n, v, d = 2100, 30_011, 136
    h, w, targets = inputs(t, n, v, d, 3)
    g = gen(8)
    hd, wd, i = h.to(DEV), w.to(DEV), targets.to(DEV)
    a, b = torch.randn(n, generator=g).to(DEV), (0.2 * torch.randn(n, generator=g)).to(DEV)
    _, entropy, lse, _, _ = learn.log_probs(hd, wd, i)
    z = hd.double() @ wd.double().t().contiguous()
    log_p = z - torch.logsumexp(z, 1)[:, None]
    p = log_p.exp()
    ent = -(p * log_p).sum(1)
    there = (i >= 0) & (i < v)
    aa = torch.where(there, a.double(), 0.0)[:, None]
    bb = b.double()[:, None]
    big = p * (aa.abs() + bb.abs() * (log_p.abs() + ent[:, None]))
    p = -p * (aa + bb * (log_p + ent[:, None]))
    at = i.clamp(0, v - 1)[:, None]
    p.scatter_add_(1, at, aa)
    big.scatter_add_(1, at, aa.abs())
    ws = torch.empty(60 << 20, dtype=torch.uint8, device=DEV)
    for more in ({}, {"workspace": ws}, {"table": False}, {"table": False, "workspace": ws}):
        dh, dw = learn.log_probs_grad(hd, wd, i, lse, a, entropy, b, **more)
        # half a step on P, and 4e-4 of its parts (logits of about 10 that are off by 1e-4 at most)
        near(dh, (p @ wd.double()).cpu(), ((half_step(t) * p.abs() + 4e-4 * big) @ wd.double().abs()).cpu(), t)
        if dw is not None:
            near(dw, (p.t().contiguous() @ hd.double()).cpu(), ((half_step(t) * p.abs() + 4e-4 * big).t().contiguous() @ hd.double().abs()).cpu(), t)
        else:
            assert more.get("table") is False


@pytest.mark.parametrize("v", [64, 300])
@pytest.mark.parametrize("size,shift", [(2, 0), (2, 12), (5, 40), (5, 100), (8, 1000), (8, 30_000)])
@pytest.mark.parametrize("scale", [1.0, 1.25, -0.7])
def test_probabilities_keep_their_bits_at_any_lse(v, size, shift, scale):
    """With the unit matrix for a table dh is P itself, and the logits are h: whatever the size of lse, p is exp(z - lse) but for the roundings of that difference."""
    n, g = 500, gen(v)
    h = (size * torch.randn(n, v, generator=g) + shift) / scale
    i = torch.randint(0, v, (n,), generator=g)
    i[::7] = -1
    a, b = torch.randn(n, generator=g), 0.3 * torch.randn(n, generator=g)
    hd, wd, id_ = h.to(DEV), torch.eye(v, device=DEV), i.to(DEV)
    _, entropy, lse, _, _ = learn.log_probs(hd, wd, id_, scale=scale)
    s = torch.tensor(scale, dtype=F32).double()
    u = h.double() * s - lse.cpu().double()[:, None]           # (lse and the entropy are given numbers here)
    p = u.exp()
    there = i >= 0
    hit = torch.zeros(n, v, dtype=torch.float64).scatter_(1, i.clamp_min(0)[:, None], 1.0) * there[:, None]
    aa = torch.where(there, a.double(), 0.0)[:, None]
    for bb in (None, b):
        bx = torch.zeros(n, 1, dtype=torch.float64) if bb is None else bb.double()[:, None]
        e = entropy.cpu().double()[:, None]
        dh, _ = learn.log_probs_grad(hd, wd, id_, lse, a.to(DEV), None if bb is None else entropy, None if bb is None else bb.to(DEV), scale=scale)
        want = s * (aa * hit - p * (aa + bx * (u + e)))
        # The exponent, log2(e) u: a factor of two roundings, its own, and 2^x by the hardware (a step); the factor of the token's: lost part (a step and a rounding), gradient, scale and
        # 1 more; the product's.  Beside p: log p and H come in two products and sums.  Products with 0 and 1 are exact.
        parts = p * (aa.abs() + bx.abs() * (u.abs() + e))
        tol = abs(s) * (parts * (3 * u.abs() + 16) * U + aa.abs() * hit * 4 * U) + 2.0 ** -126
        off = ((dh.cpu().double() - want).abs() - tol).max().item()
        assert off <= 0, "beyond the bound by %g" % off


@pytest.mark.parametrize("scale", [1e-37, 1.2e-38, 1e-40, -3e-43, 2.0 ** -149])
def test_gradients_at_the_smallest_scales(scale):
    """Factors that are no normal numbers: every row is as likely as any other, and P what a large gradient leaves of the factor."""
    n, v, d = 70, 300, 24
    h, w, targets = inputs(F32, n, v, d, 5)
    a = 1e36 * torch.randn(n, generator=gen(1))
    hd, wd, i = h.to(DEV), w.to(DEV), targets.to(DEV)
    _, _, lse, _, _ = learn.log_probs(hd, wd, i, scale=scale)
    ref = Ref(h, w, targets, torch.tensor(scale, dtype=F32).double().item())
    dh, dw = learn.log_probs_grad(hd, wd, i, lse, a.to(DEV), scale=scale)
    _grad_check(ref, a, None, F32, dh, dw)


def test_an_infinite_gradient_keeps_its_sign():
    """fp32: the row a token's infinite gradient asks for goes one way, all others the other."""
    h, w, targets = inputs(F32, 5, 40, 8, 6, ignored=False)
    h = h.abs() + 0.1
    a = torch.zeros(5)
    a[2] = math.inf
    hd, wd, i = h.to(DEV), w.to(DEV), targets.to(DEV)
    _, _, lse, _, _ = learn.log_probs(hd, wd, i)
    _, dw = learn.log_probs_grad(hd, wd, i, lse, a.to(DEV))
    others = torch.ones(40, dtype=torch.bool)
    others[targets[2]] = False
    assert (dw.cpu()[targets[2]] == math.inf).all() and (dw.cpu()[others] == -math.inf).all()


def test_gradients_are_the_differences():
    g = gen(11)
    h, w, targets = inputs(F32, 50, 90, 20, 11)
    dlogp, dentropy = torch.randn(50, generator=g), torch.randn(50, generator=g)
    _, entropy, lse, _, _ = learn.log_probs(h.to(DEV), w.to(DEV), targets.to(DEV), scale=0.5)
    dh, dw = learn.log_probs_grad(h.to(DEV), w.to(DEV), targets.to(DEV), lse, dlogp.to(DEV), entropy, dentropy.to(DEV), scale=0.5)
    wh, ww = torch.randn(h.shape, generator=g, dtype=torch.float64), torch.randn(w.shape, generator=g, dtype=torch.float64)

    def value(h, w):
        ref = Ref(h, w, targets, 0.5)
        return (ref.logp * dlogp.double() + ref.entropy * dentropy.double()).sum().item()
    h, w, e = h.double(), w.double(), 1e-4
    assert abs((dh.cpu().double() * wh).sum().item() - (value(h + e * wh, w) - value(h - e * wh, w)) / (2 * e)) < 1e-4
    assert abs((dw.cpu().double() * ww).sum().item() - (value(h, w + e * ww) - value(h, w - e * ww)) / (2 * e)) < 1e-4


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("n,v", [(70, 300), (300, 9000)])
def test_tokens_without_a_part(t, n, v):
    h, w, targets = inputs(t, n, v, 48, 9, ignored=False)
    g = gen(3)
    a, b = torch.randn(n, generator=g), torch.randn(n, generator=g)
    keep = torch.ones(n, dtype=torch.bool)
    keep[::3] = False
    b[~keep] = 0
    odd = h.clone()
    odd[~keep] = math.nan
    odd[0, 5] = math.inf
    i = torch.where(keep, targets, torch.tensor([-100])).to(DEV)
    out = []
    for x, da in ((odd, torch.where(keep, a, torch.tensor([math.nan]))), (h, a)):
        logp, entropy, lse, _, _ = learn.log_probs(x.to(DEV), w.to(DEV), i)
        out.append((logp,) + learn.log_probs_grad(x.to(DEV), w.to(DEV), i, lse, da.to(DEV), entropy, b.to(DEV)))
    for x, y in zip(*out):
        assert torch.equal(x, y)
    logp, dh, dw = out[0]
    assert (logp.cpu()[~keep] == 0).all() and (dh.cpu()[~keep] == 0).all() and torch.isfinite(dw).all()
    # a token without a target has its entropy's gradient still
    b = torch.randn(n, generator=g)
    _, entropy, lse, _, _ = learn.log_probs(h.to(DEV), w.to(DEV), i)
    dh, dw = learn.log_probs_grad(h.to(DEV), w.to(DEV), i, lse, a.to(DEV), entropy, b.to(DEV))
    _grad_check(Ref(h, w, i.cpu(), 1.0), a, b, t, dh, dw)
    none = torch.full((n,), v, device=DEV)
    dh, dw = learn.log_probs_grad(h.to(DEV), w.to(DEV), none, lse, a.to(DEV), entropy, b.to(DEV))
    _grad_check(Ref(h, w, none.cpu(), 1.0), a, b, t, dh, dw)
    # nobody has anything, and there is nobody
    dh, dw = learn.log_probs_grad(odd.to(DEV), w.to(DEV), none, lse, a.to(DEV), entropy, torch.zeros(n, device=DEV))
    assert (dh == 0).all() and (dw == 0).all()
    dh, dw = learn.log_probs_grad(h[:0].to(DEV), w.to(DEV), none[:0], lse[:0], lse[:0])
    assert dh.shape == (0, 48) and (dw == 0).all()
    assert learn.log_probs_grad(h[:0].to(DEV), w.to(DEV), none[:0], lse[:0], lse[:0], table=False)[1] is None


def test_gradient_of_impossible_rows():
    """Logits of -infinity: a probability of 0, with no part in either gradient."""
    n, v = 40, 300
    w = torch.zeros(v, 8)
    w[::3, 0] = -math.inf
    w[:, 1] = torch.linspace(-1, 1, v)
    h = torch.ones(n, 8)
    i = torch.ones(n, dtype=torch.int64)
    for t in TYPES:
        hd, wd = h.to(t).to(DEV), w.to(t).to(DEV)
        logp, entropy, lse, _, _ = learn.log_probs(hd, wd, i.to(DEV))
        _, dw = learn.log_probs_grad(hd, wd, i.to(DEV), lse, torch.ones(n, device=DEV), entropy, torch.ones(n, device=DEV))
        assert torch.isfinite(logp).all() and torch.isfinite(entropy).all() and torch.isfinite(dw).all() and (dw[::3] == 0).all()


# ---- the gradients' norm

def _many(seed, sizes, types=TYPES, size=1.0):
    g = gen(seed)
    return [(size * torch.randn(n, generator=g)).to(types[i % len(types)]).to(DEV) for i, n in enumerate(sizes)]


def _norm_ref(grads, scale):
    return abs(scale) * math.sqrt(sum((g.double() ** 2).sum().item() for g in grads))


LISTS = [[1], [0, 5, 0], [7, 8193, 16_384, 3], [8192], [1_000_003, 1, 5], [33, 1089] * 70, [1] * 129, [100_000] * 300, [3_000_000, 1000, 3_000_001]]


@pytest.mark.parametrize("sizes", LISTS, ids=lambda s: "%dx%d" % (len(s), sum(s)))
def test_norm_and_clipping(sizes):
    grads = _many(len(sizes), sizes)
    for scale in (1.0, -0.25):
        want = _norm_ref(grads, scale)
        norm = learn.grad_norm(grads, scale=scale)
        assert norm.shape == () and norm.dtype == F32 and abs(norm.item() - want) <= want * (half_step(F32) + 1e-12)
        for max_norm in (want * 0.3, want * 1.7, math.inf, 0.0):
            factor = scale * (min(1.0, max_norm / want) if want else 1.0)
            out = [torch.full_like(g, 7.0) for g in grads]
            before = [g.clone() for g in grads]
            assert torch.equal(learn.clip_grads(grads, max_norm, scale=scale, out=out), norm)
            for g, b, o in zip(grads, before, out):
                assert torch.equal(g, b)
                # the factor's own rounding, the norm's and max_norm's as fp32 numbers, the product's
                near(o, g.cpu().double() * factor, g.cpu().double().abs() * abs(factor) * 4 * U, g.dtype)
            # in place: the same
            assert torch.equal(learn.clip_grads(before, max_norm, scale=scale), norm)
            for b, o in zip(before, out):
                assert torch.equal(b, o)


def test_clipping_leaves_what_is_beside():
    flat = torch.full((50_000,), 3.0, dtype=BF16, device=DEV)
    parts = [flat[1:4], flat[5:8200], flat[10_001:30_004]]
    learn.clip_grads(parts, 1.0)
    keep = torch.ones(50_000, dtype=torch.bool)
    for a, b in ((1, 4), (5, 8200), (10_001, 30_004)):
        keep[a:b] = False
    assert (flat.cpu()[keep] == 3).all()
    assert abs(math.sqrt(sum((p.double() ** 2).sum().item() for p in parts)) - 1.0) < half_step(BF16) + 4 * U


@pytest.mark.parametrize("t", TYPES)
def test_norm_of_huge_and_tiny_values(t):
    top = torch.finfo(t).max
    for size in (top / 2, torch.finfo(t).tiny * 4, 1e-20 if t != F16 else 1e-6, 0.0):
        g = [torch.full((n,), size, dtype=t, device=DEV) for n in (3, 20_000)]
        want = _norm_ref(g, 1.0)
        got = learn.grad_norm(g).item()
        if want > torch.finfo(F32).max:
            assert got == math.inf
        else:
            assert abs(got - want) <= want * (half_step(F32) + 1e-12) + 2.0 ** -149
        if want:
            # under a norm of 1, or to it from the largest numbers: the factor is what fp32 holds
            max_norm = want / 4
            if max_norm < 3e38:
                out = [torch.empty_like(x) for x in g]
                learn.clip_grads(g, max_norm, out=out)
                for x, o in zip(g, out):
                    near(o, x.cpu().double() * 0.25, x.cpu().double().abs() * 2 * U, t)
    # a norm beyond fp32 brings finite values under max_norm still
    if t != F16:
        g = [torch.full((1000,), 3e38, dtype=t, device=DEV)]
        assert learn.clip_grads(g, 1.0).item() == math.inf
        near(g[0], torch.full((1000,), 1000 ** -0.5, dtype=torch.float64), torch.full((1000,), 8 * U), t)


@pytest.mark.parametrize("t", [F32, BF16])
@pytest.mark.parametrize("in_place", [True, False])
def test_norms_around_the_end_of_fp32(t, in_place):
    """Finite values are brought under max_norm whether or not fp32 holds their norm; an infinite value beside them leaves all as they are."""
    top = torch.finfo(F32).max
    for by, scale in ((0.9, 1.0), (1.0 + 2.0 ** -7, 1.0), (10.0, 1.0), (10.0, -2.0 ** -3), (0.9, 16.0)):
        # 100 values and 44: the norm is 12 times one of them
        grads = [torch.full((n,), by * top / 12, dtype=t, device=DEV) for n in (100, 44)]
        value = grads[0][0].double().item()
        want = 12 * value * abs(scale)
        out = [g.clone() for g in grads] if in_place else [torch.empty_like(g) for g in grads]
        norm = learn.clip_grads(out if in_place else grads, 6.0, scale=scale, out=None if in_place else out).item()
        assert norm == math.inf if want > top * (1 + U) else abs(norm - want) <= want * (half_step(F32) + 1e-12)
        for o in out:
            # (the factor's rounding, in two steps below 2^-64, and the product's)
            near(o, torch.full(o.shape, 0.5 if scale > 0 else -0.5, dtype=torch.float64), torch.full(o.shape, 4 * U), t)
        for bad in (math.inf, math.nan):
            grads[1][3] = bad
            out = [g.clone() for g in grads] if in_place else [torch.empty_like(g) for g in grads]
            norm = learn.clip_grads(out if in_place else grads, 6.0, scale=scale, out=None if in_place else out).item()
            assert norm == math.inf if bad == math.inf else math.isnan(norm)
            for o, g in zip(out, grads):
                assert torch.equal((g * scale).nan_to_num(nan=5.0), o.nan_to_num(nan=5.0))


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_norms_that_are_none(bad):
    grads = _many(4, [100, 20_000, 7])
    grads[1][12_345] = bad
    before = [g.clone() for g in grads]
    norm = learn.clip_grads(grads, 0.5)
    assert norm.isnan() if math.isnan(bad) else norm == math.inf
    assert torch.equal(learn.grad_norm(grads).isnan(), norm.isnan())
    for a, b in zip(grads, before):
        assert torch.equal(a.nan_to_num(nan=5.0), b.nan_to_num(nan=5.0))
    learn.clip_grads(grads, 0.5, scale=2.0)
    for a, b in zip(grads, before):
        assert torch.equal(a.nan_to_num(nan=5.0), (b * 2).nan_to_num(nan=5.0))


def test_norm_past_32_bits_of_values():
    n = (1 << 32) + 12_345
    g = torch.zeros(n, dtype=BF16, device=DEV)
    at = torch.tensor([0, 1 << 31, (1 << 32) - 1, 1 << 32, n - 1], device=DEV)
    g[at] = 3.0
    norm = learn.clip_grads([g], 1.0)
    assert abs(norm.item() - math.sqrt(45)) <= 7 * U
    assert (g[at].double() - 1 / math.sqrt(5)).abs().max() <= half_step(BF16) * 0.5 and int((g != 0).sum()) == 5


# ---- how they are called

def _policy_step(h, w, targets, weights, bonus, more):
    logp, entropy, lse, rows, row_logp = learn.log_probs(h, w, targets, scale=1.5, top=4)
    dh, dw = learn.log_probs_grad(h, w, targets, lse, weights, entropy, bonus, scale=1.5)
    own = more.clone()
    norm = learn.clip_grads([dh, dw, own], 0.01)
    return logp, entropy, lse, rows, row_logp, dh, dw, own, norm, learn.grad_norm([dh, dw, own])


def _policy_inputs(seed, n, v, d, t=BF16):
    g = gen(seed)
    return ((2 * torch.randn(n, d, generator=g)).to(t).to(DEV), (torch.randn(v, d, generator=g) / math.sqrt(d)).to(t).to(DEV), torch.randint(-1, v, (n,), generator=g).to(DEV),
            (torch.randn(n, generator=g) / n).to(DEV), (0.1 * torch.rand(n, generator=g) / n).to(DEV), torch.randn(777, generator=g).to(DEV))


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("n", [1, 48, 300, 5000])
def test_a_step_in_a_graph(t, n):
    state = [x.clone() for x in _policy_inputs(0, n, 1500, 64, t)]
    _policy_step(*state)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _policy_step(*state)
    for seed in range(4):
        for a, b in zip(state, _policy_inputs(seed, n, 1500, 64, t)):
            a.copy_(b)
        want = [x.clone() for x in _policy_step(*state)]
        for o in out:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b)


def test_on_another_stream():
    state = _policy_inputs(4, 300, 700, 96, F32)
    want = _policy_step(*state)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        big = torch.randn(4096, 4096, device=DEV)
        for _ in range(20):
            big = big @ big * 1e-3                   # the stream is busy: a call on another one would be in front
        late = [x.clone() for x in state]
        got = _policy_step(*late)
    side.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)


def test_two_calls_at_once():
    """Two streams, a workspace each: neither meets the other's."""
    one, two = _policy_inputs(5, 400, 9000, 64), _policy_inputs(6, 400, 9000, 64)
    want = [_policy_step(*one), _policy_step(*two)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        got = []
        for s, x in zip(streams, (one, two)):
            with torch.cuda.stream(s):
                got.append(_policy_step(*x))
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            for x, y in zip(a, b):
                assert torch.equal(x, y)


def test_refusals_of_the_binding():
    x = torch.zeros(4, 8, device=DEV)
    i = torch.zeros(4, dtype=torch.int64, device=DEV)
    f = torch.zeros(4, device=DEV)
    for call in (lambda: learn.log_probs(x, x.half(), i), lambda: learn.log_probs(x, x, i[:3]), lambda: learn.log_probs(x, x[:, :4], i), lambda: learn.log_probs(x, x, i, top=33),
                 lambda: learn.log_probs(x, x, i, top=-1), lambda: learn.log_probs(x.t(), x, i), lambda: learn.log_probs(x.double(), x.double(), i),
                 lambda: learn.log_probs(x, x, i.float()), lambda: learn.log_probs(x[0], x, i), lambda: learn.log_probs_grad(x, x, i, f, f[:2]),
                 lambda: learn.log_probs_grad(x, x, i, f.half(), f), lambda: learn.log_probs_grad(x, x, i, f, f, dentropy=f), lambda: learn.log_probs_grad(x, x, i, f, f, f[:3], f),
                 lambda: learn.log_probs_grad(x, x, i, f, f, workspace=torch.zeros(1, dtype=torch.uint8, device=DEV).expand(1 << 20)),
                 lambda: learn.grad_norm([]), lambda: learn.grad_norm([x.t()]), lambda: learn.grad_norm([i]), lambda: learn.grad_norm([x, x.cpu()]), lambda: learn.clip_grads([x], -1.0),
                 lambda: learn.clip_grads([x], math.nan), lambda: learn.clip_grads([x], 1.0, out=[]), lambda: learn.clip_grads([x], 1.0, out=[f]), lambda: learn.clip_grads([x], 1.0, out=[x.half()])):
        with pytest.raises((TypeError, ValueError)):
            call()
    # a tensor that would be written where another is
    for call in (lambda: learn.clip_grads([x, x], 1.0), lambda: learn.clip_grads([x, x.view(-1)[8:24]], 1.0), lambda: learn.clip_grads([x[:2], x[2:]], 1.0, out=[x[2:], x[:2]]),
                 lambda: learn.clip_grads([x[:3]], 1.0, out=[x[1:]]), lambda: learn.clip_grads([x.clone(), f], 1.0, out=[x, x.view(-1)[28:]])):
        with pytest.raises(knn.TagoreError, match="written"):
            call()
    learn.clip_grads([x[:2], x[2:]], 1.0)
    learn.clip_grads([x, x], 1.0, out=[x.clone(), x.clone()])            # (read twice: counted twice)
    assert abs(learn.grad_norm([x + 1, x + 1]).item() - 8.0) < 1e-6
    for scale in (math.inf, math.nan):
        with pytest.raises(knn.TagoreError, match="scale"):
            learn.grad_norm([x], scale=scale)
    logp, entropy, lse, rows, row_logp = learn.log_probs(x[:0], x, i[:0], top=3)
    assert logp.shape == entropy.shape == lse.shape == (0,) and rows.shape == row_logp.shape == (0, 3)


def test_tensors_that_require_a_gradient_are_refused():
    x, f = torch.randn(4, 8, device=DEV), torch.ones(4, device=DEV)
    i = torch.zeros(4, dtype=torch.int64, device=DEV)
    p = torch.nn.Parameter
    for call in (lambda: learn.log_probs(p(x), x, i), lambda: learn.log_probs(x, p(x), i), lambda: learn.log_probs_grad(x, p(x), i, f, f), lambda: learn.log_probs_grad(x, x, i, f, p(f)),
                 lambda: learn.grad_norm([x, p(x)]), lambda: learn.clip_grads([p(x.clone())], 1.0), lambda: learn.clip_grads([x], 1.0, out=[p(x.clone())])):
        with pytest.raises(ValueError, match="no_grad"):
            call()
        with torch.no_grad():
            call()


def test_autograd_is_told_what_is_written():
    """A tensor that a graph has kept for its backward pass: written in place, that pass refuses as it does behind torch's own operators."""
    def kept():
        x = torch.randn(1000, device=DEV, requires_grad=True)
        return x, x.exp()
    for into in (False, True):
        x, y = kept()
        other = torch.ones(30, device=DEV)
        version, beside = y._version, other._version
        with torch.no_grad():
            if into:
                learn.clip_grads([other, torch.ones(1000, device=DEV)], 0.5, out=[torch.empty(30, device=DEV), y])
            else:
                learn.clip_grads([other, y], 0.5)
        assert y._version > version and (other._version == beside) == into
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.sum().backward()
    # what is only read has not changed
    x, y = kept()
    version = y._version
    with torch.no_grad():
        learn.grad_norm([y])
        learn.clip_grads([y], 0.5, out=[torch.empty(1000, device=DEV)])
    assert y._version == version
    y.sum().backward()
    with torch.inference_mode():
        z = torch.ones(100, device=DEV)
        learn.clip_grads([z], 1.0)
    assert abs(z.norm().item() - 1) < 1e-6


def test_tangents_are_refused():
    import torch.autograd.forward_ad as forward_ad
    x, f = torch.randn(4, 8, device=DEV), torch.ones(4, device=DEV)
    i = torch.zeros(4, dtype=torch.int64, device=DEV)
    with forward_ad.dual_level():
        dual, line = forward_ad.make_dual(x, torch.ones_like(x)), forward_ad.make_dual(f, f.clone())
        for call in (lambda: learn.log_probs(dual, x, i), lambda: learn.log_probs(x, dual, i), lambda: learn.log_probs_grad(x, x, i, f, line), lambda: learn.grad_norm([x, dual]),
                     lambda: learn.clip_grads([f, dual], 1.0), lambda: learn.clip_grads([x], 1.0, out=[dual]), lambda: embed.softmax_xent(dual, x, i), lambda: embed.lookup(dual, i)):
            with pytest.raises(ValueError, match="tangent"):
                call()
        # tensors without one are taken, and a Function has them so
        want = learn.log_probs(x, x, i)[2]
        assert torch.equal(learn.log_probs(forward_ad.unpack_dual(dual).primal, x, i)[2], want)

        class Lse(torch.autograd.Function):
            @staticmethod
            def forward(ctx, h):
                return learn.log_probs(h, x, i)[2]

            @staticmethod
            def jvp(ctx, t):
                return t.sum(1)
        out = forward_ad.unpack_dual(Lse.apply(dual))
        assert torch.equal(out.primal, want) and torch.equal(out.tangent, torch.full((4,), 8.0, device=DEV))
