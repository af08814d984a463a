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
