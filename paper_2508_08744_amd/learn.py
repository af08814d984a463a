"""Python binding of include/tagore_learn.h: the operators that tune a learnt table by what it answers with.

Argument marshalling only, in the manner of ``embed``: torch supplies device memory and the current stream, the HIP library does the work,
and there is no fallback.  torch's autograd sees none of it: tensors that require a gradient are refused while gradients are recorded, and those with a tangent
of its forward mode; of the tensors that ``clip_grads`` writes it is told that they have changed.
Matrices may have any row stride (their last dimension must be contiguous); results are new contiguous tensors.
"""
from __future__ import annotations

import array
import ctypes
import math
import operator

import torch

from . import embed
from .embed import DTYPES, TagoreError, _aligned, _check, _forward_mode, _ids, _on_device, _ptr, _rows, _space, _stream, _vector  # noqa: F401

EXPORTS = ["tg_log_probs_workspace", "tg_log_probs", "tg_log_probs_grad_workspace", "tg_log_probs_grad", "tg_grad_norm_workspace", "tg_grad_norm",
           "tg_clip_grads"]

MAX_TOP = 32

_lib = None


def lib():
    """The loaded library with this header's signatures; raises if it has not been built."""
    global _lib
    if _lib is None:
        L = embed.lib()
        vp, i64, i32, f32, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_float, ctypes.c_size_t
        L.tg_log_probs_workspace.argtypes = [i64, i64, i32, i32, i32, i32]
        L.tg_log_probs.argtypes = [vp, i64, vp, i64, i32, i64, i64, i32, vp, i32, f32, i32, vp, vp, vp, vp, vp, vp, sz, vp]
        L.tg_log_probs_grad_workspace.argtypes = [i64, i64, i32, i32, i32, i32]
        L.tg_log_probs_grad.argtypes = [vp, i64, vp, i64, i32, i64, i64, i32, vp, i32, vp, vp, vp, vp, f32, vp, vp, vp, sz, vp]
        L.tg_grad_norm_workspace.argtypes = [vp, i32]
        L.tg_grad_norm.argtypes = [vp, vp, vp, i32, f32, vp, vp, sz, vp]
        L.tg_clip_grads.argtypes = [vp, vp, vp, vp, i32, f32, f32, vp, vp, sz, vp]
        for name in EXPORTS:
            if name.endswith("_workspace"):
                getattr(L, name).restype = sz
        _lib = L
    return _lib


def log_probs(h, w, targets=None, scale=1.0, top=0):
    """tg_log_probs: (logp, entropy, lse, rows, row_logp) of every row of h scored against all rows of w.

    logp: the log probability of each target, 0 where it is no row of w (None without ``targets``); rows, row_logp: the ``top`` best rows (at
    most 32) and their log probabilities, best first, n x top.
    """
    ld_h, n, d = _rows("h", h)
    ld_w, v, d_w = _rows("w", w, h.dtype)
    if d_w != d:
        raise ValueError("h and w must have rows of the same length")
    if not 0 <= top <= MAX_TOP:
        raise ValueError("top must be in 0..%d" % MAX_TOP)
    wide = 0 if targets is None else _ids("targets", targets, n)
    f32 = torch.float32
    logp = None if targets is None else h.new_empty(n, dtype=f32)
    entropy, lse = h.new_empty(n, dtype=f32), h.new_empty(n, dtype=f32)
    rows, row_logp = h.new_empty(n, top, dtype=torch.int32), h.new_empty(n, top, dtype=f32)
    t, L = DTYPES[h.dtype], lib()
    nbytes = L.tg_log_probs_workspace(n, v, d, t, top, _aligned(h, ld_h, w, ld_w))
    keep, ws = _space(nbytes, h)
    _check(L.tg_log_probs(h.data_ptr(), ld_h, w.data_ptr(), ld_w, t, n, v, d, _ptr(targets), wide, scale, top, _ptr(logp), entropy.data_ptr(),
                          lse.data_ptr(), rows.data_ptr(), row_logp.data_ptr(), ws, nbytes, _stream(h, w, targets)))
    return logp, entropy, lse, rows, row_logp


def log_probs_grad(h, w, targets, lse, dlogp, entropy=None, dentropy=None, scale=1.0, table=True, workspace=None):
    """tg_log_probs_grad: (dh, dw) from the gradients dlogp of every token's log probability and, where given, dentropy of its entropy.

    ``table=False``: dw is not formed, and None.  ``workspace``: a uint8 tensor to use instead of a new one; a smaller one makes smaller pieces
    of the table, down to what the library refuses.
    """
    ld_h, n, d = _rows("h", h)
    ld_w, v, d_w = _rows("w", w, h.dtype)
    if d_w != d:
        raise ValueError("h and w must have rows of the same length")
    wide = _ids("targets", targets, n)
    _vector("lse", lse, n, (torch.float32,))
    _vector("dlogp", dlogp, n, (torch.float32,))
    if dentropy is not None:
        if entropy is None:
            raise ValueError("the gradient of the entropy needs the entropy")
        _vector("entropy", entropy, n, (torch.float32,))
        _vector("dentropy", dentropy, n, (torch.float32,))
    else:
        entropy = None
    dh = h.new_empty(n, d)
    dw = h.new_empty(v, d) if table else None
    t, L = DTYPES[h.dtype], lib()
    if workspace is None:
        nbytes = L.tg_log_probs_grad_workspace(n, v, d, t, 1 if table else 0, _aligned(h, ld_h, w, ld_w))
        keep, ws = _space(nbytes, h)
    else:
        _on_device("workspace", workspace, (torch.uint8,), 1)
        if not workspace.is_contiguous():
            raise ValueError("workspace must be contiguous")
        ws, nbytes = workspace.data_ptr(), workspace.numel()
    _check(L.tg_log_probs_grad(h.data_ptr(), ld_h, w.data_ptr(), ld_w, t, n, v, d, targets.data_ptr(), wide, lse.data_ptr(), dlogp.data_ptr(),
                               _ptr(entropy), _ptr(dentropy), scale, dh.data_ptr(), _ptr(dw), ws, nbytes,
                               _stream(h, w, targets, lse, dlogp, entropy, dentropy, workspace)))
    return dh, dw


_REQUIRES_GRAD = operator.attrgetter("requires_grad")
_DATA_PTR, _NUMEL, _DEVICE, _CONTIGUOUS = torch.Tensor.data_ptr, torch.Tensor.numel, torch.Tensor.get_device, torch.Tensor.is_contiguous


def _tensors(name, grads):
    """The tensors' addresses, counts and types as the library takes them (whole lists at a time: 0.27 instead of 0.45 us a tensor)."""
    try:
        types = [DTYPES[g.dtype] for g in grads]
        devices = set(map(_DEVICE, grads))
        if min(devices) < 0:
            raise TypeError
    except (AttributeError, KeyError, TypeError):
        raise TypeError("%s must be CUDA tensors of %s" % (name, " or ".join(str(d) for d in DTYPES))) from None
    if not all(map(_CONTIGUOUS, grads)):
        raise ValueError("%s must be contiguous" % name)
    # the checks of _stream, which looks at a tensor at a time: one of every device, one that requires a gradient, and those with tangents
    for g in grads if len(devices) > 1 else grads[:1]:
        _stream(g)
    if torch.is_grad_enabled():
        for g in filter(_REQUIRES_GRAD, grads):
            _stream(g)
    if _forward_mode():
        _stream(*grads)
    return array.array("Q", map(_DATA_PTR, grads)), array.array("q", map(_NUMEL, grads)), array.array("i", types)


def _at(a):
    return a.buffer_info()[0]


def _list(name, grads):
    grads = list(grads)
    if not grads:
        raise ValueError("%s must hold a tensor at least" % name)
    return grads


def _norm_space(grads, counts):
    L = lib()
    nbytes = L.tg_grad_norm_workspace(_at(counts), len(grads))
    keep, ws = _space(nbytes, grads[0])
    return L, keep, ws, nbytes, grads[0].new_empty((), dtype=torch.float32)


def grad_norm(grads, scale=1.0):
    """tg_grad_norm: |scale| times the norm of all values of a list of tensors together, a tensor of one fp32 value."""
    grads = _list("grads", grads)
    at, counts, types = _tensors("grads", grads)
    L, keep, ws, nbytes, norm = _norm_space(grads, counts)
    _check(L.tg_grad_norm(_at(at), _at(counts), _at(types), len(grads), scale, norm.data_ptr(), ws, nbytes, _stream()))
    return norm


def clip_grads(grads, max_norm, scale=1.0, out=None):
    """tg_clip_grads: the tensors times scale, and brought under max_norm together; in their own place, or into those of ``out``.

    The norm of grads * scale before that is returned, a tensor of one fp32 value.  Where a value is infinite or NaN (the norm then is, too) the tensors
    are but multiplied with scale; finite values are brought under max_norm whatever their norm, also where it is beyond fp32 and returned as infinity.
    """
    if math.isnan(max_norm) or max_norm < 0:
        raise ValueError("max_norm must not be below 0")
    grads = _list("grads", grads)
    at, counts, types = _tensors("grads", grads)
    to = at
    if out is not None:
        out = _list("out", out)
        if len(out) != len(grads):
            raise ValueError("out must have a tensor for every gradient")
        to, out_counts, out_types = _tensors("out", out)
        if out_counts != counts or out_types != types:
            raise ValueError("out must have the gradients' sizes and types")
    L, keep, ws, nbytes, norm = _norm_space(grads, counts)
    _check(L.tg_clip_grads(_at(at), _at(to), _at(counts), _at(types), len(grads), max_norm, scale, norm.data_ptr(), ws, nbytes, _stream()))
    torch.autograd.graph.increment_version(grads if out is None else out)
    return norm
