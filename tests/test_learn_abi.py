"""CPU-only checks of include/tagore_learn.h: exports, refusals before anything is enqueued, workspaces, and host loops at the ends of the sizes."""
import ctypes
import os
import re
import subprocess
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = ctypes.c_void_p(256)          # never followed: every call below is refused first, or has nothing to do
ODD = ctypes.c_void_p(264)
BIG = 1 << 62


def test_library_exports_every_declared_symbol():
    from paper_2508_08744_amd import learn
    text = open(os.path.join(ROOT, "include", "tagore_learn.h")).read()
    names = sorted(set(re.findall(r"\b(tg_[a-z0-9_]+)\s*\(", re.sub(r"/\*.*?\*/", "", text, flags=re.S))))
    assert sorted(learn.EXPORTS) == names and len(names) == 7
    for name in names:
        assert hasattr(learn.lib(), name), name


def _refused(call, good, bad):
    """Every (position, value) of `bad` alone makes the call invalid."""
    from paper_2508_08744_amd import learn
    for at, value in bad:
        a = list(good)
        a[at] = value
        assert getattr(learn.lib(), call)(*a) == -1, (call, at, value)
        assert learn.lib().tg_last_error()


def test_log_probs_refusals():
    from paper_2508_08744_amd import learn
    L = learn.lib()
    good = [P, 64, P, 64, 1, 10, 1000, 64, P, 1, 1.0, 8, P, P, P, P, P, P, BIG, None]
    _refused("tg_log_probs", good, [(0, None), (1, 63), (2, None), (3, 63), (4, 3), (4, -1), (5, -1), (5, 1 << 28), (6, 0), (6, 1 << 30), (7, 0), (7, 8193), (9, 2), (11, -1),
                                    (11, 33), (12, None), (13, None), (14, None), (15, None), (16, None), (17, None), (17, ODD), (18, 100)])
    good = [P, 64, P, 64, 1, 10, 1000, 64, P, 1, P, P, P, P, 1.0, P, P, P, BIG, None]
    _refused("tg_log_probs_grad", good, [(0, None), (1, 63), (2, None), (3, 63), (4, 3), (5, -1), (6, 0), (7, 0), (8, None), (9, 2), (10, None), (11, None), (12, None), (15, None),
                                         (17, None), (17, ODD), (18, 100)])
    # nothing to do
    assert L.tg_log_probs(None, 64, None, 64, 1, 0, 1000, 64, None, 1, 1.0, 8, None, None, None, None, None, None, 0, None) == 0
    assert L.tg_log_probs_grad(None, 64, None, 64, 1, 0, 1000, 64, None, 1, None, None, None, None, 1.0, None, None, None, 0, None) == 0


def test_log_probs_workspaces():
    from paper_2508_08744_amd import learn
    f, g = learn.lib().tg_log_probs_workspace, learn.lib().tg_log_probs_grad_workspace
    for bad in ((-1, 1000, 64, 1, 8, 1), (10, 0, 64, 1, 8, 1), (10, 1000, 8193, 1, 8, 1), (10, 1000, 64, 3, 8, 1), (10, 1000, 64, 1, 33, 1), (10, 1000, 64, 1, -1, 1),
                (10, 1000, 64, 1, 8, 4), (0, 1000, 64, 1, 8, 1)):
        assert f(*bad) == 0
    for bad in ((-1, 1000, 64, 1, 1, 1), (10, 1000, 64, 1, 2, 1), (10, 1000, 64, 1, 1, -1), (0, 1000, 64, 1, 1, 1)):
        assert g(*bad) == 0
    n, v, d = 48, 100_000, 96
    h, w = n * d * 2, v * d * 2
    both, table, tokens, none = (f(n, v, d, 1, 8, a) for a in (1, 2, 3, 0))
    assert h <= table - both <= h + 256 and w <= tokens - both <= w + 256 and h + w <= none - both <= h + w + 512
    assert f(n, v, 97, 1, 8, 1) == f(n, v, 97, 1, 8, 0)              # rows of such a length are copied wherever they start
    # the best rows cost a byte a logit at most, and no more than a GiB at a time
    assert f(n, v, d, 1, 8, 1) - f(n, v, d, 1, 0, 1) <= n * v + 64 * 1024
    assert f(1 << 20, 100_000, 64, 1, 8, 1) < (1 << 30) + (1 << 28)
    # without the table's gradient, no more than with it
    for n in (1, 40, 999, 8192):
        assert 0 < g(n, 37_511, 512, 2, 0, 1)


def test_the_gradients_workspace_without_the_tables():
    """Neither with nor without the table's gradient is the other's bound; they differ by dh's parts, 64 of n x d fp32 at most, and the pieces' alignment."""
    from paper_2508_08744_amd import learn
    g = learn.lib().tg_log_probs_grad_workspace
    more = 0
    for n in (1, 7, 40, 64, 65, 300, 999, 8192):
        for v, d in ((1, 8), (5000, 50), (37_511, 512), (131_072, 1024), (1_000_003, 96)):
            for dtype in (0, 1, 2):
                without, with_it = g(n, v, d, dtype, 0, 1), g(n, v, d, dtype, 1, 1)
                assert without > 0 and with_it > 0 and abs(without - with_it) <= 64 * n * d * 4 + 512
                more += without > with_it
    assert more > 0


def _lists(pointers, counts, types):
    n = len(counts)
    return (ctypes.c_void_p * n)(*pointers), (ctypes.c_int64 * n)(*counts), (ctypes.c_int32 * n)(*types)


def test_norm_refusals():
    from paper_2508_08744_amd import learn
    L = learn.lib()
    at, counts, types = _lists([1024, 4096, None], [100, 50, 0], [0, 1, 2])
    good = [at, counts, types, 3, 1.0, P, P, BIG, None]
    nan, inf = float("nan"), float("inf")
    _refused("tg_grad_norm", good, [(0, None), (1, None), (2, None), (3, -1), (3, (1 << 20) + 1), (4, nan), (4, inf), (5, None), (6, None), (6, ODD), (7, 8)])
    clip = [at, at, counts, types, 3, 1.0, 1.0, P, P, BIG, None]
    _refused("tg_clip_grads", clip, [(0, None), (1, None), (2, None), (3, None), (4, -1), (5, -1.0), (5, nan), (6, -inf), (7, None), (8, None), (8, ODD), (9, 8)])
    for pointers, c, t in (([1024, 4096], [100, -1], [0, 1]), ([1024, 4096], [100, 1 << 40], [0, 1]), ([1024, 4096], [1, 1], [0, 3]), ([1024, None], [1, 1], [0, 1]),
                           ([1026, 4096], [1, 1], [0, 1]), ([1024, 4097], [1, 1], [0, 1])):
        lists = _lists(pointers, c, t)
        assert L.tg_grad_norm(*lists, 2, 1.0, P, P, BIG, None) == -1 and L.tg_clip_grads(lists[0], lists[0], *lists[1:], 2, 1.0, 1.0, P, P, BIG, None) == -1
    f = L.tg_grad_norm_workspace
    assert f(counts, -1) == 0 and f(counts, (1 << 20) + 1) == 0 and f(None, 3) == 0 and f(_lists([], [1 << 40], [])[1], 1) == 0
    assert 8 * 1024 <= f(counts, 3) <= 16 * 1024


def test_clipping_writes_no_tensor_where_another_is():
    from paper_2508_08744_amd import learn
    L = learn.lib()

    def call(grads, out, counts, types):
        g, c, t = _lists(grads, counts, types)
        o = _lists(out, counts, types)[0]
        # (a workspace that is too small: what is refused for its ranges is refused before)
        assert L.tg_clip_grads(g, o, c, t, len(grads), 1.0, 1.0, P, P, 8, None) == -1
        return b"written" in L.tg_last_error()
    A, B, C = 1 << 20, 1 << 21, 1 << 22
    assert not call([A, B], [A, B], [10, 10], [0, 1])
    assert not call([A, B], [C, C + 40], [10, 10], [0, 1])
    assert not call([A, A], [C, B], [10, 10], [0, 0])                     # read twice
    assert not call([A, A + 40], [A, A + 40], [10, 10], [0, 0])           # back to back
    assert not call([A, A], [A, C], [10, 0], [0, 0])                      # of none
    assert call([A, A], [A, A], [10, 10], [0, 0])
    assert call([A, A], [A, C], [10, 10], [0, 0])                         # the one's place is read by the other
    assert call([A, B], [B, A], [10, 10], [0, 0])
    assert call([A], [A + 4], [10], [0]) and call([A + 4], [A], [10], [0])
    assert call([A, B], [C, C + 36], [10, 10], [0, 0]) and call([A, B], [C + 36, C], [10, 10], [0, 0])
    assert call([A, B, C], [A, B, A + 38], [10, 10, 10], [0, 0, 1])
    assert call([A, B, C], [A, B - 16, C], [100, 2, 2], [0, 1, 1]) is False and call([A, B, C], [A, B - 2, C], [100, 2, 2], [0, 1, 1])


def test_binding_refuses_host_tensors():
    from paper_2508_08744_amd import learn
    x, i, s = torch.zeros((8, 16)), torch.zeros(8, dtype=torch.int64), torch.zeros(8)
    for call in (lambda: learn.log_probs(x, x, i), lambda: learn.log_probs_grad(x, x, i, s, s), lambda: learn.grad_norm([x]), lambda: learn.clip_grads([x], 1.0),
                 lambda: learn.grad_norm([])):
        with pytest.raises((TypeError, ValueError)):
            call()


CALLS = """
import ctypes
from paper_2508_08744_amd import learn
L, P, BIG = learn.lib(), ctypes.c_void_p(256), 1 << 62
ANY = (-4, 0)                       # TG_ERR_HIP: nothing was wrong with the arguments
%s
print("back")
"""
ENDS = {
    "rows": """
for dtype in (0, 1, 2):
    for n in (1, 33, 65, 129, 300, 5000):
        for v in ((1 << 29), (1 << 29) + 1, (1 << 30) - 1):
            for top in (0, 32):
                rc = L.tg_log_probs(P, 4, P, 4, dtype, n, v, 4, P, 1, 1.0, top, P, P, P, P, P, P, BIG, None)
                assert rc == -4, rc
""",
    "tokens": """
for dtype in (0, 1, 2):
    for n in ((1 << 28) - 1, (1 << 27) + 3):
        for v in (1, 40, 700):
            for top in (0, 32):
                rc = L.tg_log_probs(P, 8, P, 8, dtype, n, v, 8, P, 0, 1.0, top, P, P, P, P, P, P, BIG, None)
                assert rc == -4, rc
""",
    "tensors": """
n = 1 << 20
at, out, counts, types = (ctypes.c_void_p * n)(), (ctypes.c_void_p * n)(), (ctypes.c_int64 * n)(), (ctypes.c_int32 * n)()
for i in range(n):
    at[i] = out[i] = 1024 + 64 * i
    counts[i] = i % 7
assert L.tg_grad_norm_workspace(counts, n) < 1 << 20
assert L.tg_clip_grads(at, out, counts, types, n, 1.0, 1.0, P, P, BIG, None) == -4
counts[0] = (1 << 40) - 1
at[0] = out[0] = 1 << 43
counts[1] = (1 << 40) - 1
at[1] = out[1] = 1 << 45
assert L.tg_clip_grads(at, out, counts, types, n, 1.0, 1.0, P, P, BIG, None) == -4
assert L.tg_grad_norm(at, counts, types, 2, 1.0, P, P, BIG, None) == -4
""",
}


@pytest.mark.parametrize("what", sorted(ENDS))
def test_calls_of_the_largest_sizes_come_back(what):
    """Where no device is visible every launch in them fails, and the call has to come back."""
    env = dict(os.environ, HIP_VISIBLE_DEVICES="-1", PYTHONPATH=ROOT)
    r = subprocess.run([sys.executable, "-c", CALLS % ENDS[what]], cwd=ROOT, env=env, timeout=100, capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.split()[-1:] == ["back"], r.stdout + r.stderr
