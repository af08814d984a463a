"""The operators of include/tagore_embed.h where values, sizes or arguments leave the ordinary: tiny, huge and infinite values, targets that
share a row or have one alone, tables of many rows, operands of uneven alignment, tensors that require a gradient.

Tolerances are bounds, from the roundings that a result goes through (half a step of its type, fp32 chains times 2^-24)."""
import math

import pytest
import torch

from paper_2508_08744_amd import embed

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
U = 2.0 ** -24


def half_step(t):
    return torch.finfo(t).eps / 2


# ---- 8-bit rows of small numbers

@pytest.mark.parametrize("d", [8, 77, 512, 4099])
@pytest.mark.parametrize("t,tops", [(BF16, (3e-36, 4e-37, 3.5e-37, 1e-37, 1.2e-38, 3e-39, 1e-40)), (F32, (3e-36, 1e-37, 1e-39, 1e-40)), (F16, (6e-8, 1e-6, 1e-4, 60000.0))])
def test_rows_of_small_numbers_on_the_grid(t, tops, d):
    g = torch.Generator().manual_seed(d)
    x = torch.rand(len(tops), d, generator=g) * 2 - 1
    x[:, 0] = 1.0
    x[:, 1::5] = 0.0
    x = (x.double() * torch.tensor(tops, dtype=torch.float64)[:, None]).to(t)
    q, scale = embed.quantize_rows(x.to(DEV))
    q, scale, z = q.cpu().double(), scale.cpu().double(), x.double()
    top = z.abs().amax(1) / 127
    # (the scale is rounded to fp32, among whose subnormal numbers the step is 2^-149)
    assert ((scale - top).abs() <= top * 2 * U + 2.0 ** -150).all() and (scale > 0).all()
    assert ((z / scale[:, None]).clamp(-127, 127) - q).abs().max() <= 0.5 + 1e-9
    assert (q[z == 0] == 0).all() and (q.abs().amax(1) == 127).all()


# ---- many rows


@pytest.mark.parametrize("n", [7, 70])
def test_losses_over_more_than_half_of_2_to_the_30_rows(n):
    """fp32 rows in tiles of 64: more tiles along the table than one launch has."""
    v, d = (1 << 29) + 1000, 4
    w = torch.zeros(v, d, device=DEV)
    far = torch.tensor([0, 63, 1 << 28, (1 << 29) - 1, 1 << 29, (1 << 29) + 64, v - 1], device=DEV)
    w[far] = torch.tensor([[20.0, 0, 0, 0], [21, 1, 0, 0], [0, 22, 0, 0], [21, 1, 1, 1], [22, 2, 0, 1], [0, 0, 24, 0], [0, 0, 0, 25]], device=DEV)
    h = torch.rand(n, d, generator=torch.Generator().manual_seed(n)).to(DEV)
    targets = far[torch.arange(n, device=DEV) % 7]
    targets[5] = 12345
    loss, lse = embed.softmax_xent(h, w, targets)
    z = h.double() @ w[far].double().t().contiguous()
    want = torch.log(torch.exp(z).sum(1) + (v - 7))
    z_t = (h.double() * w[targets].double()).sum(1)
    # a tile of equal terms is exact; a lane of the join adds a 256th of the tiles one after another; the far rows' logits and exponents: 400
    tol = (v / 64 / 256 + 400) * U
    assert ((lse.double() - want).abs() <= tol).all() and ((loss.double() - (want - z_t)).abs() <= 2 * tol).all()
