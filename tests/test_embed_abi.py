"""CPU-only checks of include/tagore_embed.h: exports, and refusals before anything is enqueued."""
import ctypes
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = ctypes.c_void_p(256)          # never followed: every call below is refused first, or has nothing to do
ODD = ctypes.c_void_p(264)
BIG = 1 << 62


def test_library_exports_every_declared_symbol():
    from paper_2508_08744_amd import embed
    text = open(os.path.join(ROOT, "include", "tagore_embed.h")).read()
    names = sorted(set(re.findall(r"\b(tg_[a-z0-9_]+)\s*\(", re.sub(r"/\*.*?\*/", "", text, flags=re.S))))
    assert sorted(embed.EXPORTS) == names and len(names) == 15
    for name in names:
        assert hasattr(embed.lib(), name), name


def _refused(call, good, bad, says=None):
    """Every (position, value) of `bad` alone makes the call invalid."""
    from paper_2508_08744_amd import embed
    for at, value in bad:
        a = list(good)
        a[at] = value
        assert getattr(embed.lib(), call)(*a) == -1, (call, at, value)
        assert embed.lib().tg_last_error()


def test_lookup_refusals():
    from paper_2508_08744_amd import embed
    good = [P, 64, 0, 1000, 64, P, 1, 10, 1.0, P, None]
    _refused("tg_embed_lookup", good, [(0, None), (1, 63), (2, 3), (2, -1), (3, 0), (3, 1 << 30), (4, 0), (4, 65537), (5, None), (6, 2), (7, -1),
                                       (7, 1 << 30), (9, None)])
    assert embed.lib().tg_embed_lookup(None, 64, 0, 1000, 64, None, 1, 0, 1.0, None, None) == 0        # no ids: nothing to do
    good = [P, 64, 1, P, 0, 10, 1000, 64, 1.0, 0, P, 0, P, BIG, None]
    _refused("tg_embed_lookup_grad", good, [(0, None), (1, 63), (2, 3), (3, None), (4, 2), (5, -1), (6, 0), (7, 0), (9, 2), (10, None), (11, 2), (11, 3),
                                            (12, None), (12, ODD), (13, 100)])
    f = embed.lib().tg_embed_lookup_grad_workspace
    assert f(0, 10, 8) == 0 and f(-1, 10, 8) == 0 and f(5, 0, 8) == 0 and f(5, 10, 0) == 0
    assert f(8192, 10, 8) < f(8193, 10, 8) and f(1 << 29, (1 << 30) - 1, 64) > 1 << 34


def test_norm_refusals():
    from paper_2508_08744_amd import embed
    nan = float("nan")
    _refused("tg_add_rms_norm", [P, 64, P, 64, P, 1, 10, 64, 1e-6, P, P, P, None],
             [(0, None), (1, 63), (3, 63), (4, None), (5, 3), (6, -1), (6, 1 << 30), (7, 0), (7, 8193), (8, -1.0), (8, nan), (9, None), (10, None)])
    _refused("tg_add_rms_norm_q8", [P, 64, P, 64, P, 1, 10, 64, 1e-6, P, P, P, None],
             [(0, None), (1, 63), (3, 63), (4, None), (5, 3), (6, -1), (7, 0), (8, float("inf")), (9, None), (10, None), (11, None)])
    _refused("tg_add_rms_norm_grad", [P, 64, P, 64, P, 64, P, P, 1, 10, 64, P, P, P, BIG, None],
             [(0, None), (1, 63), (3, 63), (4, None), (5, 63), (6, None), (7, None), (8, 3), (9, -1), (10, 8193), (11, None), (12, None), (13, None),
              (13, ODD), (14, 10)])
    _refused("tg_quantize_rows", [P, 64, 0, 10, 64, P, P, None], [(0, None), (1, 63), (2, 7), (3, -1), (4, 0), (5, None), (6, None)])
    _refused("tg_dequantize_rows", [P, P, 10, 64, 0, P, None], [(0, None), (1, None), (2, -1), (3, 0), (4, 3), (5, None)])
    assert embed.lib().tg_add_rms_norm(None, 64, None, 0, None, 1, 0, 64, 1e-6, None, None, None, None) == 0


def test_product_refusals():
    from paper_2508_08744_amd import embed
    _refused("tg_matmul_q8", [P, P, P, P, None, 10, 20, 64, P, 0, None, 0, None],
             [(0, None), (1, None), (2, None), (3, None), (5, -1), (6, 0), (6, 1 << 30), (7, 0), (7, 65537), (8, None), (9, 3)])
    # rows that have to be copied need a workspace
    _refused("tg_matmul_q8", [P, P, P, P, None, 100, 20, 300, P, 0, P, BIG, None], [(10, None), (10, ODD), (11, 100)])
    _refused("tg_matmul_q8", [P, P, ODD, P, None, 100, 20, 320, P, 0, P, BIG, None], [(10, None), (11, 100)])
    f = embed.lib().tg_matmul_q8_workspace
    assert f(100, 20, 320, 1) == 0 and f(100, 20, 320, 0) >= 120 * 320 and f(100, 20, 300, 1) >= 120 * 304 and f(100, 20, 320, 2) == 0
    assert f(64, 20, 300, 0) == 0 and f(100, 20, 250, 0) == 0          # few tokens and short rows are read as they are
    assert embed.lib().tg_matmul_q8(None, None, None, None, None, 0, 20, 64, None, 0, None, 0, None) == 0


def test_softmax_xent_refusals():
    from paper_2508_08744_amd import embed
    _refused("tg_softmax_xent", [P, 64, P, 64, 1, 10, 1000, 64, P, 1, 1.0, P, P, P, BIG, None],
             [(0, None), (1, 63), (2, None), (3, 63), (4, 3), (5, -1), (5, 1 << 30), (6, 0), (7, 0), (7, 8193), (8, None), (9, 2), (11, None), (12, None),
              (13, None), (13, ODD), (14, 100)])
    _refused("tg_softmax_xent_grad", [P, 64, P, 64, 1, 10, 1000, 64, P, 1, P, P, 1.0, P, P, P, BIG, None],
             [(0, None), (1, 63), (2, None), (3, 63), (4, 3), (5, -1), (6, 0), (7, 0), (8, None), (9, 2), (10, None), (11, None), (13, None), (14, None),
              (15, None), (15, ODD), (16, 100)])
    f, g = embed.lib().tg_softmax_xent_workspace, embed.lib().tg_softmax_xent_grad_workspace
    assert f(0, 10, 8, 0, 1) == 0 and g(0, 10, 8, 0, 1) == 0 and f(5, 10, 8, 3, 1) == 0 and f(5, 10, 8, 0, 5) == 0
    # a table that has to be copied costs its bytes
    assert f(64, 100_000, 96, 1, 0) - f(64, 100_000, 96, 1, 1) >= 100_000 * 192
    assert g(64, 100_000, 50, 1, 1) >= 100_000 * 112


def test_binding_refuses_host_tensors():
    from paper_2508_08744_amd import embed
    x = torch.zeros((8, 16))
    w = torch.zeros(16)
    i = torch.zeros(8, dtype=torch.int64)
    q = torch.zeros((8, 16), dtype=torch.int8)
    s = torch.zeros(8)
    for call in (lambda: embed.lookup(x, i), lambda: embed.lookup_grad(x, i, 10), lambda: embed.add_rms_norm(x, w), lambda: embed.quantize_rows(x),
                 lambda: embed.add_rms_norm_grad(x, x, w, s), lambda: embed.add_rms_norm_q8(x, w), lambda: embed.dequantize_rows(q, s),
                 lambda: embed.matmul_q8(q, s, q, s), lambda: embed.softmax_xent(x, x, i), lambda: embed.softmax_xent_grad(x, x, i, s, s)):
        with pytest.raises((TypeError, ValueError)):
            call()
