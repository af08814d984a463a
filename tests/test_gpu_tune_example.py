"""examples/learn_and_index.py: its steps of tuning by rewards, and the answers that they are drawn from."""
import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu


def _example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "learn_and_index.py")
    spec = importlib.util.spec_from_file_location("learn_and_index", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _logits(table, weight, item):
    x = table[item] * math.sqrt(table.shape[1])
    return (x * torch.rsqrt((x * x).mean(1, keepdim=True) + 1e-6) * weight) @ table.t()


@pytest.mark.parametrize("max_norm", [math.inf, 0.01])
def test_a_tuning_steps_gradients(max_norm):
    m = _example()
    gen = torch.Generator(device="cuda").manual_seed(4)
    n, v, d = 700, 900, 40
    table = 0.5 * torch.randn(v, d, generator=gen, device="cuda")
    weight = 1 + 0.1 * torch.randn(d, generator=gen, device="cuda")
    item, answer = (torch.randint(0, v, (n,), generator=gen, device="cuda") for _ in range(2))
    answer[::9] = -1
    gain, bonus = torch.randn(n, generator=gen, device="cuda") / n, torch.rand(n, generator=gen, device="cuda") / n
    dtable, dweight, norm = m.tune_step(table, weight, item, answer, gain, bonus, max_norm)
    a, b = table.cpu().double().requires_grad_(), weight.cpu().double().requires_grad_()
    log_p = torch.log_softmax(_logits(a, b, item.cpu()), 1)
    there = answer.cpu() >= 0
    logp = log_p.gather(1, answer.cpu().clamp_min(0)[:, None])[:, 0]
    value = -(gain.cpu().double() * logp)[there].sum() + (bonus.cpu().double()[:, None] * log_p.exp() * log_p).sum()
    value.backward()
    whole = math.sqrt((a.grad ** 2).sum() + (b.grad ** 2).sum())
    factor = min(1.0, max_norm / whole)
    # fp32 throughout: six operators, each within a few hundred roundings of 2^-24 of the largest entry
    assert abs(norm.item() - whole) <= 2000 * 2.0 ** -24 * whole
    for got, ref in ((dtable, a.grad), (dweight, b.grad)):
        assert (got.cpu().double() - factor * ref).abs().max() <= 2000 * 2.0 ** -24 * factor * ref.abs().max()


def test_answers_are_the_best_rows():
    m = _example()
    gen = torch.Generator(device="cuda").manual_seed(5)
    table = torch.randn(3000, 24, generator=gen, device="cuda")
    weight = torch.ones(24, device="cuda")
    item = torch.randint(0, 3000, (200,), generator=gen, device="cuda")
    rows, logp = m.answers(table, weight, item, top=9)
    # the normed rows as the operator gives them: its roundings are those of the logits' other side
    from paper_2508_08744_amd import embed
    y, _, _ = embed.add_rms_norm(embed.lookup(table, item, scale=math.sqrt(24)), weight)
    log_p = torch.log_softmax(y.cpu().double() @ table.cpu().double().t(), 1)
    best, at = torch.sort(log_p, dim=1, descending=True, stable=True)
    assert torch.equal(rows.cpu().long(), at[:, :9])
    # logits of up to 40 whose terms' magnitudes sum to 100 at most: 27 roundings of these
    assert (logp.cpu().double() - best[:, :9]).abs().max() <= 2 * 27 * 100 * 2.0 ** -24 + 400 * 2.0 ** -24


def test_tuning_runs():
    m = _example()
    gen = torch.Generator(device="cuda").manual_seed(6)
    table = (torch.randn(2000, 64, generator=gen, device="cuda") / 8).bfloat16()
    weight = torch.ones(64, device="cuda", dtype=torch.bfloat16)
    tuned, w, shares = m.tune(table, weight, 20, 1024, 3)
    assert tuned.shape == table.shape and tuned.dtype == torch.bfloat16 and torch.isfinite(tuned).all() and torch.isfinite(w).all() and shares.shape == (3,)
    assert not torch.equal(tuned, table) and m.tune(table, weight, 20, 1024, 0)[2] is None
