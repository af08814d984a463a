"""CPU-only: calls of include/tagore_embed.h that are refused, and what the workspaces cost."""
import ctypes
import importlib.util

import torch

P, Q, R = (ctypes.c_void_p(256 * i) for i in (1, 2, 3))          # never followed: every call below is refused


def test_norms_in_place_of_rows_that_are_apart():
    """out_r has rows of d: written over x or the residual, it would meet rows still to be read if those are further apart."""
    from paper_2508_08744_amd import embed
    L = embed.lib()
    for x, ld_x, res, ld_res in ((R, 72, Q, 64), (Q, 64, R, 72), (R, 72, R, 64), (R, 72, R, 72)):
        assert L.tg_add_rms_norm(x, ld_x, res, ld_res, P, 1, 10, 64, 1e-6, P, R, P, None) == -1
        assert b"back to back" in L.tg_last_error()
        assert L.tg_add_rms_norm_q8(x, ld_x, res, ld_res, P, 1, 10, 64, 1e-6, P, P, R, None) == -1
        assert b"back to back" in L.tg_last_error()


def test_binding_without_torchs_private_names(monkeypatch):
    """A build of torch without them: the module is imported, and asks for the stream by the public names."""
    from paper_2508_08744_amd import embed
    for name in ("_cuda_getDevice", "_cuda_getCurrentRawStream"):
        if hasattr(torch._C, name):
            monkeypatch.delattr(torch._C, name)
    spec = importlib.util.spec_from_file_location("paper_2508_08744_amd.embed_of_another_torch", embed.__file__)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)

    class Stream:
        def __init__(self, device):
            self.cuda_stream = 100 + device
    monkeypatch.setattr(torch.cuda, "current_stream", Stream)
    assert m._device is torch.cuda.current_device and m._raw_stream(3) == 103


def test_workspaces_copy_only_the_odd_operand():
    from paper_2508_08744_amd import embed
    f, g = embed.lib().tg_softmax_xent_workspace, embed.lib().tg_softmax_xent_grad_workspace
    n, v, d = 48, 100_000, 96
    h, w = n * d * 2, v * d * 2
    both, table, tokens, none = (f(n, v, d, 1, a) for a in (1, 2, 3, 0))
    assert h <= table - both <= h + 256 and w <= tokens - both <= w + 256 and h + w <= none - both <= h + w + 512
    assert g(n, v, d, 1, 1) == g(n, v, d, 1, 2) and w <= g(n, v, d, 1, 3) - g(n, v, d, 1, 1) <= w + 256 and g(n, v, d, 1, 3) == g(n, v, d, 1, 0)
    assert f(n, v, d, 1, 4) == 0 and f(n, v, d, 1, -1) == 0 and g(n, v, d, 1, 4) == 0
    assert f(n, v, 97, 1, 1) == f(n, v, 97, 1, 0)                # rows of such a length are copied wherever they start
