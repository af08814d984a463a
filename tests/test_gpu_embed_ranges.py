"""The operators of include/tagore_embed.h at the ends of their ranges: values, row ends and token counts at which a kernel goes another way."""
import pytest
import torch

from paper_2508_08744_amd import embed

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -24


@pytest.mark.parametrize("d", [64, 77, 2056, 8000])
def test_8_bit_norm_of_products_beyond_fp32(d):
    g = torch.Generator().manual_seed(d)
    x = (0.5 + torch.rand(9, d, generator=g)) * torch.where(torch.rand(9, d, generator=g) < 0.5, -1.0, 1.0)
    x *= torch.tensor([2e38, 1e38, 1.0, 1e-20, 1e-37, 1e-30, 1e25, 1e-25, 0.0])[:, None]
    x = x.bfloat16()
    for factor in (16.0, 1e-10, 1.0):
        w = (factor * (1 + torch.rand(d, generator=g))).bfloat16()
        z = x.double()
        y = z / torch.sqrt((z * z).mean(1, keepdim=True)) * w.double()
        q, scale, _ = embed.add_rms_norm_q8(x.to(DEV), w.to(DEV), eps=0.0)
        q, scale = q.cpu().double(), scale.cpu().double()
        assert torch.isnan(scale[8]) and (q[8] == 0).all()
        top = y[:8].abs().amax(1) / 127
        assert ((scale[:8] - top).abs() <= top * 2 * U).all()
        assert ((y[:8] / scale[:8, None] - q[:8]).abs() <= 0.5 + 1e-9).all()


@pytest.mark.parametrize("m,n,k", [(1, 1, 3), (5, 129, 17), (130, 700, 65), (203, 4099, 100), (70, 1000, 127), (300, 515, 191), (64, 2050, 255)])
@pytest.mark.parametrize("t", [torch.float32, torch.float16])
def test_short_products_up_to_the_last_byte(m, n, k, t):
    """Rows of any length whose last one ends where the memory given ends: what lies behind is not zero, and what is stored ends where the output does."""
    g = torch.Generator().manual_seed(m + n + k)
    flat = torch.full((n * k + 64,), 77, dtype=torch.int8)
    flat[:n * k] = torch.randint(-127, 128, (n * k,), generator=g).to(torch.int8)
    b = flat.to(DEV)[:n * k].view(n, k)
    a = torch.randint(-127, 128, (m, k), generator=g).to(torch.int8)
    sa, sb, bias = torch.rand(m, generator=g), torch.rand(n, generator=g), torch.randn(n, generator=g)
    for add in (bias, None):
        got = embed.matmul_q8(a.to(DEV), sa.to(DEV), b, sb.to(DEV), bias=None if add is None else add.to(DEV), out_dtype=t).cpu().double()
        terms = (a.double() @ flat[:n * k].view(n, k).double().t()) * sa.double()[:, None] * sb.double()
        want = terms if add is None else terms + add.double()
        # the sum's rounding to fp32, two products and an addition, then the type's half step
        bound = 3 * U * terms.abs() + U * (terms.abs() * (1 + 3 * U) + (0 if add is None else add.double().abs()))
        # (a value that the type does not hold becomes infinite: half a step beyond its largest)
        most = torch.finfo(t).max * (1 + torch.finfo(t).eps / 4)
        beyond = want.abs() - bound > most
        assert torch.equal(got[beyond], torch.copysign(torch.full_like(got[beyond], float("inf")), want[beyond]))
        held = want.abs() + bound < most
        assert ((got - want).abs() <= bound + torch.finfo(t).eps / 2 * (want.abs() + bound) + torch.finfo(t).tiny)[held].all()


@pytest.mark.parametrize("n,v,d", [(6144, 1023, 8), (6145, 1024, 4), (65_537, 70_001, 3), (262_144, 2_000_000, 2), (262_145, 1_048_576, 5), (600_000, 1000, 12)])
def test_lookup_gradient_of_many_tokens(n, v, d):
    """The sorts' borders, in whole numbers: every sum is exact, so the order does not show, and the counts do."""
    g = torch.Generator().manual_seed(n)
    ids = torch.randint(-3, v + 3, (n,), generator=g)
    ids[::3] = v // 2                                    # a third of the tokens are one row's
    x = torch.randint(-8, 9, (n, d), generator=g).float()
    there = (ids >= 0) & (ids < v)
    want = torch.zeros(v, d).index_add_(0, ids[there], x[there])
    got = embed.lookup_grad(x.to(DEV), ids.to(DEV), v)
    assert torch.equal(got.cpu(), want)
    out = torch.ones(v, d, device=DEV)
    embed.lookup_grad(x.to(DEV), ids.int().to(DEV), v, out=out)
    assert torch.equal(out.cpu(), want + 1)
    for t in (torch.bfloat16, torch.float16):
        x8 = x.clone()
        x8[there & (ids == v // 2)] = 0                  # (the large sums need more than the type's bits)
        want8 = torch.zeros(v, d).index_add_(0, ids[there], x8[there])
        got = embed.lookup_grad(x8.to(t).to(DEV), ids.to(DEV), v).cpu()
        assert torch.equal(got, want8.to(t))


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [1, 3, 7, 9, 13, 257, 511])
def test_lookup_gradient_adds_shared_columns_once(t, d):
    """Rows that end inside a piece: the last one shares columns with the one before."""
    g = torch.Generator().manual_seed(d)
    ids = torch.randint(0, 40, (500,), generator=g)
    x = torch.randint(-3, 4, (500, d), generator=g).float()
    out = torch.randint(-5, 6, (40, d), generator=g).float()
    want = out + torch.zeros(40, d).index_add_(0, ids, x)
    got = out.to(DEV)
    embed.lookup_grad(x.to(t).to(DEV), ids.to(DEV), 40, out=got)
    assert torch.equal(got.cpu(), want)
    got = out.to(t).to(DEV)
    embed.lookup_grad(x.to(t).to(DEV), ids.to(DEV), 40, out=got)
    assert torch.equal(got.cpu(), want.to(t))
