"""CPU-only: the entry points' host code at the ends of the documented sizes.  The calls run where no device is visible: every launch in them
fails, and the call has to come back."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CALLS = """
import ctypes
from paper_2508_08744_amd import embed
L, P, BIG = embed.lib(), ctypes.c_void_p(256), 1 << 62
for dtype in (0, 1, 2):
    for n in (1, 33, 65, 129, 300, 5000):
        for v in %s:
            for d in (4, 8):
                rc = L.tg_softmax_xent(P, d, P, d, dtype, n, v, d, P, 1, 1.0, P, P, P, BIG, None)
                assert rc == -4, rc                   # TG_ERR_HIP: nothing was wrong with the arguments
print("back")
"""


@pytest.mark.parametrize("rows", ["(1 << 29,)", "((1 << 29) + 1,)", "((1 << 29) + 64,)", "((1 << 30) - 1,)"])
def test_losses_over_large_tables_come_back(rows):
    """More tiles along the table than a launch has work-items for: the launches are split, and end."""
    env = dict(os.environ, HIP_VISIBLE_DEVICES="-1", PYTHONPATH=ROOT)
    r = subprocess.run([sys.executable, "-c", CALLS % rows], cwd=ROOT, env=env, timeout=100, capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.split()[-1:] == ["back"], r.stdout + r.stderr
