"""examples/learn_and_index.py: the operators together, on a table small enough for a second of learning."""
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


def _mean_loss(table, weight, item, target, scale):
    x = table[item] * math.sqrt(table.shape[1])
    y = x * torch.rsqrt((x * x).mean(1, keepdim=True) + 1e-6) * weight
    z = y @ table.t() * scale
    there = target >= 0
    return (torch.logsumexp(z, 1) - z.gather(1, target.clamp_min(0)[:, None])[:, 0])[there].sum() / there.sum()


def test_a_steps_gradients():
    m = _example()
    gen = torch.Generator(device="cuda").manual_seed(3)
    item, target = m.sessions(gen, 700, 900, 9)
    table = torch.randn(900, 40, generator=gen, device="cuda")
    weight = 1 + 0.1 * torch.randn(40, generator=gen, device="cuda")
    loss, dtable, dweight = m.step(table, weight, item, target, 0.7)
    a, b = table.cpu().double().requires_grad_(), weight.cpu().double().requires_grad_()
    want = _mean_loss(a, b, item.cpu(), target.cpu(), 0.7)
    want.backward()
    # fp32 throughout: five operators, each within a few hundred roundings of 2^-24 of the largest entry
    for got, ref in ((loss, want.detach()), (dtable, a.grad), (dweight, b.grad)):
        assert (got.cpu().double() - ref).abs().max() <= 2000 * 2.0 ** -24 * ref.abs().max()


def test_what_is_learnt_is_found():
    m = _example()
    items, topics = 2000, 20
    table, weight, losses = m.learn(items, 64, 4096, 60, topics)
    assert losses[0] > math.log(items) - 0.5 and losses[-1] < math.log(items / topics) + 1.0
    queries = torch.arange(0, items, 37, device=table.device)
    scores, ids, graph = m.serve(table, weight, queries)
    rows = (table.float() * torch.rsqrt((table.float() ** 2).mean(1, keepdim=True) + 1e-6) * weight.float()).cpu().double()
    want = rows[queries.cpu()] @ rows.t()
    # half a step of the grid on either side: max|y| / 254 of every value of the other row
    step = rows.abs().amax(1) / 254
    size = rows.abs().sum(1)
    bound = step[queries.cpu()][:, None] * size + size[queries.cpu()][:, None] * step + 64 * step[queries.cpu()][:, None] * step
    assert ((scores.cpu().double() - want).abs() <= 1.01 * bound).all()
    near = (ids % topics == (torch.arange(items, device=ids.device) % topics)[:, None]).float().mean()
    assert near > 0.9 and graph.shape == (items, 16)
