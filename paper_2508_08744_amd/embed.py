"""Python binding of include/tagore_embed.h: the operators that learn and serve the vectors a graph is built over.

Argument marshalling only, like ``knn``: torch supplies device memory and the current stream, the HIP library does the work, and there
is no fallback.  Training calls come in pairs, an operator and its gradient; nothing is kept between them but what the caller passes on.
torch's autograd sees none of it: tensors that require a gradient are refused while gradients are recorded.
Matrices may have any row stride (their last dimension must be contiguous); results are new contiguous tensors.
"""
from __future__ import annotations

import ctypes

import torch

from . import knn
from .knn import TagoreError  # noqa: F401  (what a refused call raises)

DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}

EXPORTS = ["tg_embed_lookup", "tg_embed_lookup_grad_workspace", "tg_embed_lookup_grad", "tg_add_rms_norm", "tg_add_rms_norm_grad_workspace",
           "tg_add_rms_norm_grad", "tg_add_rms_norm_q8", "tg_quantize_rows", "tg_dequantize_rows", "tg_matmul_q8_workspace", "tg_matmul_q8",
           "tg_softmax_xent_workspace", "tg_softmax_xent", "tg_softmax_xent_grad_workspace", "tg_softmax_xent_grad"]

_lib = None


def lib():
    """The loaded library with this header's signatures; raises if it has not been built."""
    global _lib
    if _lib is None:
        L = knn.lib()
        vp, i64, i32, f32, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_float, ctypes.c_size_t
        L.tg_embed_lookup.argtypes = [vp, i64, i32, i64, i32, vp, i32, i64, f32, vp, vp]
        L.tg_embed_lookup_grad_workspace.argtypes = [i64, i64, i32]
        L.tg_embed_lookup_grad.argtypes = [vp, i64, i32, vp, i32, i64, i64, i32, f32, i32, vp, i32, vp, sz, vp]
        L.tg_add_rms_norm.argtypes = [vp, i64, vp, i64, vp, i32, i64, i32, f32, vp, vp, vp, vp]
        L.tg_add_rms_norm_grad_workspace.argtypes = [i64, i32]
        L.tg_add_rms_norm_grad.argtypes = [vp, i64, vp, i64, vp, i64, vp, vp, i32, i64, i32, vp, vp, vp, sz, vp]
        L.tg_add_rms_norm_q8.argtypes = [vp, i64, vp, i64, vp, i32, i64, i32, f32, vp, vp, vp, vp]
        L.tg_quantize_rows.argtypes = [vp, i64, i32, i64, i32, vp, vp, vp]
        L.tg_dequantize_rows.argtypes = [vp, vp, i64, i32, i32, vp, vp]
        L.tg_matmul_q8_workspace.argtypes = [i64, i64, i32, i32]
        L.tg_matmul_q8.argtypes = [vp, vp, vp, vp, vp, i64, i64, i32, vp, i32, vp, sz, vp]
        L.tg_softmax_xent_workspace.argtypes = [i64, i64, i32, i32, i32]
        L.tg_softmax_xent.argtypes = [vp, i64, vp, i64, i32, i64, i64, i32, vp, i32, f32, vp, vp, vp, sz, vp]
        L.tg_softmax_xent_grad_workspace.argtypes = [i64, i64, i32, i32, i32]
        L.tg_softmax_xent_grad.argtypes = [vp, i64, vp, i64, i32, i64, i64, i32, vp, i32, vp, vp, f32, vp, vp, vp, sz, vp]
        for name in EXPORTS:
            if name.endswith("_workspace"):
                getattr(L, name).restype = sz
        _lib = L
    return _lib


def _check(rc):
    if rc != 0:
        raise TagoreError("tagore_knn error %d: %s" % (rc, lib().tg_last_error().decode()))


# The current device and stream without an object around them, 0.2 instead of 3.1 us of a call that takes 8: names of torch's own, so
# where a build of it has others, the public ones are taken.
_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda device: torch.cuda.current_stream(device).cuda_stream)


def _stream(*tensors):
    """The current stream's handle; refuses tensors that are not on its device, or whose gradient would go missing."""
    device = _device()
    for t in tensors:
        if t is not None:
            if t.get_device() != device:
                raise ValueError("a tensor is not on the current device")
            if t.requires_grad and torch.is_grad_enabled():
                raise ValueError("a tensor requires a gradient, and these calls record none: call them under torch.no_grad() or from a "
                                 "torch.autograd.Function, with the gradient's own call in its backward")
    return _raw_stream(device)


def _on_device(name, t, dtypes, dim):
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype in dtypes and t.dim() == dim):
        raise TypeError("%s must be a %d-D CUDA tensor of %s" % (name, dim, " or ".join(str(d) for d in dtypes)))


def _rows(name, t, like=None, shape=None):
    """A matrix whose rows are contiguous: the distance between them, and its shape."""
    _on_device(name, t, DTYPES if like is None else (like,), 2)
    n, d = s = t.shape
    if shape is not None and s != shape:
        raise ValueError("%s must have shape %s" % (name, tuple(shape)))
    ld, one = t.stride()
    if one != 1 and d > 1 or ld < d and n > 1:
        raise ValueError("%s must have contiguous rows that do not overlap" % name)
    return (ld if n > 1 else d), n, d


def _vector(name, t, n, dtypes):
    _on_device(name, t, dtypes, 1)
    if t.numel() != n or n > 1 and t.stride(0) != 1:
        raise ValueError("%s must be contiguous and have %d elements" % (name, n))


def _ids(name, t, n=None):
    """Whether the ids have 64 bits."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype in (torch.int64, torch.int32) and t.is_contiguous()):
        raise TypeError("%s must be a contiguous int32 or int64 CUDA tensor" % name)
    if n is not None and t.numel() != n:
        raise ValueError("%s must have %d elements" % (name, n))
    return 1 if t.dtype == torch.int64 else 0


def _space(nbytes, like):
    """A workspace and its address; the memory is the current stream's, as the calls are."""
    if nbytes == 0:
        return None, None
    ws = like.new_empty(nbytes, dtype=torch.uint8)
    return ws, ws.data_ptr()


def _ptr(t):
    return None if t is None else t.data_ptr()


def _aligned(h, ld_h, w, ld_w):
    """Which of two matrices starts at a multiple of 16 bytes, with rows such a multiple (of at most 1 MiB) apart: 1 both, 2 w, 3 h, 0 none."""
    e = h.element_size()
    far = 1 << 20
    h_is = not (h.data_ptr() | ld_h * e) % 16 and ld_h * e <= far
    if not (w.data_ptr() | ld_w * e) % 16 and ld_w * e <= far:
        return 1 if h_is else 2
    return 3 if h_is else 0


def lookup(table, ids, scale=1.0):
    """tg_embed_lookup: scale * table[ids], zeros where an id is no row of the table; the shape of ids and the rows' length."""
    ld, v, d = _rows("table", table)
    wide = _ids("ids", ids)
    out = table.new_empty(*ids.shape, d)
    _check(lib().tg_embed_lookup(table.data_ptr(), ld, DTYPES[table.dtype], v, d, ids.data_ptr(), wide, ids.numel(), scale, out.data_ptr(),
                                 _stream(table, ids)))
    return out


def lookup_grad(grad, ids, n_rows, scale=1.0, out=None):
    """tg_embed_lookup_grad: the gradient of ``lookup`` with respect to its table of ``n_rows`` rows.

    grad has a row for every id (its leading dimensions may be those of ids).  With ``out`` (a contiguous fp32 tensor, or one of
    grad's type) the sums are added to it and only rows with a token are touched; without, a new tensor of grad's type is returned.
    """
    wide = _ids("ids", ids)
    n = ids.numel()
    if isinstance(grad, torch.Tensor) and 2 != grad.dim() == ids.dim() + 1 and grad.shape[:-1] == ids.shape:
        grad = grad.reshape(-1, grad.shape[-1])
    ld, rows, d = _rows("grad", grad)
    if rows != n:
        raise ValueError("grad must have a row for every id")
    add = out is not None
    if add:
        _rows("out", out, shape=(n_rows, d))
        if out.dtype not in (torch.float32, grad.dtype) or not out.is_contiguous():
            raise TypeError("out must be contiguous and float32 or of the gradient's type")
    else:
        out = grad.new_empty(n_rows, d)
    L = lib()
    nbytes = L.tg_embed_lookup_grad_workspace(n, n_rows, d)
    keep, ws = _space(nbytes, grad)
    _check(L.tg_embed_lookup_grad(grad.data_ptr(), ld, DTYPES[grad.dtype], ids.data_ptr(), wide, n, n_rows, d, scale, int(add), out.data_ptr(),
                                  DTYPES[out.dtype], ws, nbytes, _stream(grad, ids, out)))
    return out


def add_rms_norm(x, weight, residual=None, eps=1e-6):
    """tg_add_rms_norm: (y, r, rstd) with r = x + residual (x itself where there is none) and y = r rstd weight."""
    ld, n, d = _rows("x", x)
    _vector("weight", weight, d, (x.dtype,))
    y = x.new_empty(n, d)
    rstd = x.new_empty(n, dtype=torch.float32)
    r, ld_res, out_r = x, 0, None
    if residual is not None:
        ld_res, _, _ = _rows("residual", residual, x.dtype, x.shape)
        r = x.new_empty(n, d)
        out_r = r.data_ptr()
    _check(lib().tg_add_rms_norm(x.data_ptr(), ld, _ptr(residual), ld_res, weight.data_ptr(), DTYPES[x.dtype], n, d, eps, y.data_ptr(), out_r,
                                 rstd.data_ptr(), _stream(x, weight, residual)))
    return y, r, rstd


def add_rms_norm_grad(dy, r, weight, rstd, dr=None):
    """tg_add_rms_norm_grad: (dx, dweight) from the gradients dy of y and dr of r; dx is the residual's gradient as well."""
    ld_r, n, d = _rows("r", r)
    ld_dy, _, _ = _rows("dy", dy, r.dtype, r.shape)
    ld_dr = 0 if dr is None else _rows("dr", dr, r.dtype, r.shape)[0]
    _vector("weight", weight, d, (r.dtype,))
    _vector("rstd", rstd, n, (torch.float32,))
    dx = r.new_empty(n, d)
    dw = r.new_empty(d)
    L = lib()
    nbytes = L.tg_add_rms_norm_grad_workspace(n, d)
    keep, ws = _space(nbytes, r)
    _check(L.tg_add_rms_norm_grad(dy.data_ptr(), ld_dy, _ptr(dr), ld_dr, r.data_ptr(), ld_r, weight.data_ptr(), rstd.data_ptr(), DTYPES[r.dtype],
                                  n, d, dx.data_ptr(), dw.data_ptr(), ws, nbytes, _stream(dy, dr, r, weight, rstd)))
    return dx, dw


def add_rms_norm_q8(x, weight, residual=None, eps=1e-6):
    """tg_add_rms_norm_q8: (q, scale, r), the normed rows as int8 with a scale each, and the residual stream."""
    ld, n, d = _rows("x", x)
    _vector("weight", weight, d, (x.dtype,))
    q = x.new_empty(n, d, dtype=torch.int8)
    scale = x.new_empty(n, dtype=torch.float32)
    r, ld_res, out_r = x, 0, None
    if residual is not None:
        ld_res, _, _ = _rows("residual", residual, x.dtype, x.shape)
        r = x.new_empty(n, d)
        out_r = r.data_ptr()
    _check(lib().tg_add_rms_norm_q8(x.data_ptr(), ld, _ptr(residual), ld_res, weight.data_ptr(), DTYPES[x.dtype], n, d, eps, q.data_ptr(),
                                    scale.data_ptr(), out_r, _stream(x, weight, residual)))
    return q, scale, r


def quantize_rows(x):
    """tg_quantize_rows: (q, scale), the rows as int8 with a scale each."""
    ld, n, d = _rows("x", x)
    q = x.new_empty(n, d, dtype=torch.int8)
    scale = x.new_empty(n, dtype=torch.float32)
    _check(lib().tg_quantize_rows(x.data_ptr(), ld, DTYPES[x.dtype], n, d, q.data_ptr(), scale.data_ptr(), _stream(x)))
    return q, scale


def _codes(name, q, scale):
    _on_device(name, q, (torch.int8,), 2)
    if not q.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    _vector(name + "_scale", scale, q.shape[0], (torch.float32,))
    return q.shape


def dequantize_rows(q, scale, dtype=torch.float32):
    """tg_dequantize_rows: q * scale, rounded to dtype."""
    n, d = _codes("q", q, scale)
    if dtype not in DTYPES:
        raise TypeError("dtype must be float32, bfloat16 or float16")
    out = q.new_empty(n, d, dtype=dtype)
    _check(lib().tg_dequantize_rows(q.data_ptr(), scale.data_ptr(), n, d, DTYPES[dtype], out.data_ptr(), _stream(q, scale)))
    return out


def matmul_q8(a, a_scale, b, b_scale, bias=None, out_dtype=torch.float32):
    """tg_matmul_q8: (a * a_scale) @ (b * b_scale).T (+ bias) with an exact integer sum; a: m x k tokens, b: n x k channels, int8."""
    m, k = _codes("a", a, a_scale)
    n, k_b = _codes("b", b, b_scale)
    if k_b != k:
        raise ValueError("a and b must have rows of the same length")
    if bias is not None:
        _vector("bias", bias, n, (torch.float32,))
    if out_dtype not in DTYPES:
        raise TypeError("out_dtype must be float32, bfloat16 or float16")
    out = a.new_empty(m, n, dtype=out_dtype)
    L = lib()
    aligned = 0 if (a.data_ptr() | b.data_ptr()) % 16 else 1
    nbytes = L.tg_matmul_q8_workspace(m, n, k, aligned)
    keep, ws = _space(nbytes, a)
    _check(L.tg_matmul_q8(a.data_ptr(), a_scale.data_ptr(), b.data_ptr(), b_scale.data_ptr(), _ptr(bias), m, n, k, out.data_ptr(),
                          DTYPES[out_dtype], ws, nbytes, _stream(a, a_scale, b, b_scale, bias)))
    return out


def softmax_xent(h, w, targets, scale=1.0):
    """tg_softmax_xent: (loss, lse) of every row of h scored against all rows of w; 0 where a target is no row of w."""
    ld_h, n, d = _rows("h", h)
    ld_w, v, d_w = _rows("w", w, h.dtype)
    if d_w != d:
        raise ValueError("h and w must have rows of the same length")
    wide = _ids("targets", targets, n)
    loss = h.new_empty(n, dtype=torch.float32)
    lse = h.new_empty(n, dtype=torch.float32)
    t, L = DTYPES[h.dtype], lib()
    nbytes = L.tg_softmax_xent_workspace(n, v, d, t, _aligned(h, ld_h, w, ld_w))
    keep, ws = _space(nbytes, h)
    _check(L.tg_softmax_xent(h.data_ptr(), ld_h, w.data_ptr(), ld_w, t, n, v, d, targets.data_ptr(), wide, scale, loss.data_ptr(), lse.data_ptr(),
                             ws, nbytes, _stream(h, w, targets)))
    return loss, lse


def softmax_xent_grad(h, w, targets, lse, dloss, scale=1.0, workspace=None):
    """tg_softmax_xent_grad: (dh, dw) from the gradient dloss of every token's loss.  ``workspace``: a uint8 tensor to use instead of
    a new one; a smaller one makes smaller pieces of the table, down to what the library refuses."""
    ld_h, n, d = _rows("h", h)
    ld_w, v, d_w = _rows("w", w, h.dtype)
    if d_w != d:
        raise ValueError("h and w must have rows of the same length")
    wide = _ids("targets", targets, n)
    _vector("lse", lse, n, (torch.float32,))
    _vector("dloss", dloss, n, (torch.float32,))
    dh = h.new_empty(n, d)
    dw = h.new_empty(v, d)
    t, L = DTYPES[h.dtype], lib()
    if workspace is None:
        nbytes = L.tg_softmax_xent_grad_workspace(n, v, d, t, _aligned(h, ld_h, w, ld_w))
        keep, ws = _space(nbytes, h)
    else:
        _on_device("workspace", workspace, (torch.uint8,), 1)
        if not workspace.is_contiguous():
            raise ValueError("workspace must be contiguous")
        ws, nbytes = workspace.data_ptr(), workspace.numel()
    _check(L.tg_softmax_xent_grad(h.data_ptr(), ld_h, w.data_ptr(), ld_w, t, n, v, d, targets.data_ptr(), wide, lse.data_ptr(), dloss.data_ptr(),
                                  scale, dh.data_ptr(), dw.data_ptr(), ws, nbytes, _stream(h, w, targets, lse, dloss, workspace)))
    return dh, dw
