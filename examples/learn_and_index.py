"""Learn the rows of a table, serve them in 8 bits and index them: the operators of ``embed`` and a graph of ``knn`` as they go together.

Synthetic sessions: items belong to topics, a session's next item is mostly one of the same topic.  A row is learnt for every item by
predicting the next one: the item's row is looked up, normed and scored against all rows of the table by a softmax cross entropy, whose
gradients go back through the norm and the lookup to the one table.  Then the normed rows are put on an 8-bit grid, a few of them are scored against all by the
integer product, and the k-NN graph of the rows is built and pruned.

    python examples/learn_and_index.py [--items 20000] [--dim 128] [--tokens 8192] [--steps 60]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2508_08744_amd import embed, knn  # noqa: E402


def sessions(gen, tokens, items, topics):
    """(item, next item) pairs; one pair in twenty is padding."""
    item = torch.randint(0, items, (tokens,), generator=gen, device=gen.device)
    other = torch.randint(0, items // topics, (tokens,), generator=gen, device=gen.device) * topics + item % topics
    return item, torch.where(torch.rand(tokens, generator=gen, device=gen.device) < 0.05, -1, other)


def step(table, weight, item, target, scale):
    """One pass there and back: the mean loss, and the gradients of the table and of the norm's weight."""
    root = math.sqrt(table.shape[1])
    x = embed.lookup(table, item, scale=root)
    y, r, rstd = embed.add_rms_norm(x, weight)
    loss, lse = embed.softmax_xent(y, table, target, scale=scale)
    count = (target >= 0).sum().clamp_min(1).float()
    dloss = (1.0 / count).expand(loss.shape[0]).contiguous()
    dy, dtable = embed.softmax_xent_grad(y, table, target, lse, dloss, scale=scale)
    dx, dweight = embed.add_rms_norm_grad(dy, r, weight, rstd)
    embed.lookup_grad(dx, item, table.shape[0], scale=root, out=dtable)          # added to the softmax's share
    return loss.sum() / count, dtable, dweight


def learn(items, dim, tokens, steps, topics=50, rate=0.02, seed=0, device="cuda"):
    """The learnt table (bf16), the norm's weight and the losses of all steps (Adam's rule on fp32 copies)."""
    gen = torch.Generator(device=device).manual_seed(seed)
    master = [torch.randn(items, dim, generator=gen, device=device) / math.sqrt(dim), torch.ones(dim, device=device)]
    first = [torch.zeros_like(p) for p in master]
    second = [torch.zeros_like(p) for p in master]
    losses = []
    for i in range(1, steps + 1):
        item, target = sessions(gen, tokens, items, topics)
        loss, *grads = step(master[0].bfloat16(), master[1].bfloat16(), item, target, 1.0)
        losses.append(loss)
        for p, m, v, g in zip(master, first, second, grads):
            g = g.float()
            m.lerp_(g, 0.1)
            v.lerp_(g * g, 0.01)
            p.sub_(rate * (m / (1 - 0.9 ** i)) / ((v / (1 - 0.99 ** i)).sqrt() + 1e-8))
    return master[0].bfloat16(), master[1].bfloat16(), torch.stack(losses)


def serve(table, weight, queries, k=32):
    """The queries' scores against all rows from 8-bit rows, and the pruned k-NN graph of the normed rows."""
    q, scale, _ = embed.add_rms_norm_q8(table, weight)
    scores = embed.matmul_q8(q[queries], scale[queries], q, scale)
    rows, _, _ = embed.add_rms_norm(table, weight)
    ids, _ = knn.knn_build(rows.float(), k, "l2", iters=6, seed=1)
    return scores, ids, knn.prune_rank(ids, k // 2)


def main():
    a = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("items", 20_000), ("dim", 128), ("tokens", 8192), ("steps", 60)):
        a.add_argument("--" + name, type=int, default=value)
    a = a.parse_args()
    topics = 50
    table, weight, losses = learn(a.items, a.dim, a.tokens, a.steps, topics)
    print("loss %.3f -> %.3f (the topics alone: %.3f)" % (losses[0], losses[-1], math.log(a.items / topics)))
    queries = torch.arange(0, a.items, max(1, a.items // 200), device=table.device)
    scores, ids, graph = serve(table, weight, queries)
    best = scores.scatter(1, queries[:, None], -math.inf).topk(10, dim=1).indices
    same = (best % topics == (queries % topics)[:, None]).float().mean()
    near = (ids % topics == (torch.arange(a.items, device=ids.device) % topics)[:, None]).float().mean()
    print("8-bit scores: %.3f of the ten best are of the query's topic; graph: %.3f of the neighbours; pruned to %d a row" % (same, near, graph.shape[1]))


if __name__ == "__main__":
    main()
