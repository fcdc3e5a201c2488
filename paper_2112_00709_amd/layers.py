"""Operators of a network's last layers (include/fb_layers.h): argument marshalling only.

What lies on the network's side of the objective: layer norm, affine layers with bias, activation and residual, and log
probabilities of given tokens with entropy and best alternatives, each with its gradient.  The functions carry the names of
the C entry points; like the rest of the binding they only check and pass on their arguments, and there is no CPU fallback.
``paper_2112_00709_amd.autograd`` has them as differentiable functions.

Rows are frames: a tensor ``[..., width]`` is taken as rows of ``width`` elements, any distance apart, the elements of a row
contiguous.  Row distances and addresses need no alignment.  Types: float32, bfloat16, float16.
"""
from __future__ import annotations

import ctypes
from typing import Optional

import paper_2112_00709_amd as _base

from . import FBError, _check  # noqa: F401  (FBError: what a failing call raises)

F32, BF16, F16 = 0, 1, 2
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
TOP_MAX = 64

# every symbol include/fb_layers.h declares
SYMBOLS = ["fb_layer_norm", "fb_layer_norm_grad_workspace_bytes", "fb_layer_norm_grad", "fb_affine_workspace_bytes", "fb_affine",
           "fb_affine_grad_workspace_bytes", "fb_affine_grad", "fb_token_logprobs_workspace_bytes", "fb_token_logprobs",
           "fb_token_logprobs_grad"]

_lib = None
torch = None                     # loaded with the library, see lib()
_types = {}
_raw_stream = None               # device index -> address of its current stream
_current_device = None


def lib() -> ctypes.CDLL:
    """The built library with these calls' signatures (fails loudly when it has not been built)."""
    global _lib, torch, _raw_stream, _current_device
    if _lib is None:
        L = _base.lib()
        vp, i32, i64, f32, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
        L.fb_layer_norm.argtypes = [vp, i64, vp, vp, i32, i64, i64, i32, f32, vp, i64, vp, vp, vp]
        L.fb_layer_norm_grad_workspace_bytes.argtypes = [i64, i64]
        L.fb_layer_norm_grad.argtypes = [vp, i64, vp, i64, vp, vp, vp, i32, i64, i64, i32, vp, i64, vp, vp, vp, sz, vp]
        L.fb_affine_workspace_bytes.argtypes = [vp, i64, vp, i64, i64, i64, i64, i32]
        L.fb_affine.argtypes = [vp, i64, vp, i64, vp, vp, i64, i64, i64, i64, i32, i32, vp, i64, i32, vp, i64, vp, sz, vp]
        L.fb_affine_grad_workspace_bytes.argtypes = [vp, i64, i32, vp, i64, vp, i64, i64, i64, i64, i32, i32]
        L.fb_affine_grad.argtypes = [vp, i64, i32, vp, i64, vp, i64, vp, i64, i64, i64, i64, i32, i32, vp, i64, vp, vp, vp, sz, vp]
        L.fb_token_logprobs_workspace_bytes.argtypes = [i64, i64, i32, i32]
        L.fb_token_logprobs.argtypes = [vp, i64, vp, i64, i64, i32, i32, vp, vp, vp, vp, vp, vp, sz, vp]
        L.fb_token_logprobs_grad.argtypes = [vp, i64, vp, vp, vp, vp, vp, i64, i64, i32, vp, i64, vp]
        for name in SYMBOLS:
            getattr(L, name).restype = sz if name.endswith("_bytes") else ctypes.c_int
        import torch as t
        torch = t
        _types.update({t.float32: F32, t.bfloat16: BF16, t.float16: F16})
        # the stream's address without the object around it, which takes as long to make as a kernel launch
        _raw_stream = getattr(t._C, "_cuda_getCurrentRawStream", None) or (lambda device: t.cuda.current_stream(device).cuda_stream)
        # (asked for beside a tensor on a GPU only: the runtime has been set up)
        _current_device = getattr(t._C, "_cuda_getDevice", None) or t.cuda.current_device
        _lib = L
    return _lib


def _type(t, what: str) -> int:
    code = _types.get(t.dtype)
    if code is None:
        raise ValueError(f"{what} must be float32, bfloat16 or float16")
    return code


def _rows(t, what: str, width: Optional[int] = None, dtype=None, lead=None, device: Optional[int] = None):
    """-> (address, row distance, rows, width, device) of [..., width] as rows; device None: it has to be the current one."""
    on = t.get_device()
    if on < 0 or on != (_current_device() if device is None else device) or t.dim() < 1:
        raise ValueError(f"{what} must be a tensor of at least one dimension on the current CUDA device")
    shape = t.shape
    w = shape[-1]
    if width is not None and w != width:
        raise ValueError(f"{what} must have rows of {width} elements")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{what} must be {dtype}")
    if lead is not None and shape[:-1] != lead:
        raise ValueError(f"{what} must have the same rows as the first argument")
    n = t.numel() // w if w else 0
    if t.is_contiguous():
        return t.data_ptr(), w, n, w, on
    if w > 1 and t.stride(-1) != 1:
        raise ValueError(f"the elements of a row of {what} must be contiguous")
    ld = seen = 0                                 # the leading dimensions have to be one walk over the rows
    for size, step in zip(reversed(shape[:-1]), reversed(t.stride()[:-1])):
        if size == 1:
            continue
        if seen == 0:
            ld, seen = step, size
        elif step != ld * seen:
            raise ValueError(f"the rows of {what} must lie at one distance")
        else:
            seen *= size
    if seen == 0:
        ld = w
    if ld < w and n > 1:
        raise ValueError(f"the rows of {what} must not overlap")
    return t.data_ptr(), ld, n, w, on


def _vector(t, what: str, n: int, dtypes, device: int):
    if t is None:
        return None
    if t.dtype not in dtypes or t.numel() != n or t.get_device() != device or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous tensor of {n} elements of {' or '.join(str(d) for d in dtypes)} on the first argument's device")
    return t.data_ptr()


def _out(like, shape, dtype):
    t = like.new_empty(shape, dtype=dtype)
    if _base.POISON_NEW_BUFFERS:
        t.view(torch.uint8).fill_(255)
    return t


def _out_like(t, dtype=None):
    """An output of t's shape and type, contiguous (where t is too by the shorter way: a third of a small call is allocations)."""
    if _base.POISON_NEW_BUFFERS or not t.is_contiguous():
        return _out(t, t.shape, dtype or t.dtype)
    return torch.empty_like(t, dtype=dtype)


def _floats(n: int, like, shape):
    """n float32 outputs of one shape in one allocation, as tensors of their own (.data): as views of one tensor they could not be
    changed in place where gradients are recorded."""
    return [t.data for t in _out(like, (n, *shape), torch.float32).unbind(0)]


def _workspace(n: int, like):
    if n == 0:
        return None, None
    ws = _out(like, (n,), torch.uint8)
    return ws, ws.data_ptr()


def fb_layer_norm(x, weight=None, bias=None, eps: float = 1e-5, want_stats: bool = False):
    """-> y like x, or with want_stats (y, mean, rstd), the latter float32 of x's leading shape.

    ``x`` [..., H]; ``weight``, ``bias`` [H], float32 or of x's type (both of one)."""
    L = lib()
    code = _type(x, "x")
    px, ldx, R, H, dev = _rows(x, "x")
    wt = weight if weight is not None else bias
    wtype = F32 if wt is None else _type(wt, "weight")
    if weight is not None and bias is not None and weight.dtype != bias.dtype:
        raise ValueError("weight and bias must have one type")
    types = torch.float32, x.dtype
    pw, pb = _vector(weight, "weight", H, types, dev), _vector(bias, "bias", H, types, dev)
    y = _out_like(x)
    mean = rstd = pm = pr = None
    if want_stats:
        mean, rstd = _floats(2, x, x.shape[:-1])
        pm, pr = mean.data_ptr(), rstd.data_ptr()
    _check(L.fb_layer_norm(px, ldx, pw, pb, wtype, R, H, code, eps, y.data_ptr(), H, pm, pr, _raw_stream(dev)))
    return (y, mean, rstd) if want_stats else y


def fb_layer_norm_grad(dy, x, mean, rstd, weight=None, want_dx: bool = True, want_dweight: bool = True, want_dbias: bool = True):
    """-> (dx like x, dweight [H] float32, dbias [H] float32), None in the place of one that is not wanted.

    ``dy`` like x; ``mean``, ``rstd``: as fb_layer_norm returned them."""
    L = lib()
    code = _type(x, "x")
    px, ldx, R, H, dev = _rows(x, "x")
    pdy, lddy, _, _, _ = _rows(dy, "dy", H, x.dtype, x.shape[:-1], dev)
    pm, pr = _vector(mean, "mean", R, (torch.float32,), dev), _vector(rstd, "rstd", R, (torch.float32,), dev)
    wtype = F32 if weight is None else _type(weight, "weight")
    pw = _vector(weight, "weight", H, (torch.float32, x.dtype), dev)
    dx = _out_like(x) if want_dx else None
    dw = _out(x, (H,), torch.float32) if want_dweight else None
    db = _out(x, (H,), torch.float32) if want_dbias else None
    need = int(L.fb_layer_norm_grad_workspace_bytes(R, H)) if want_dweight or want_dbias else 0
    ws, pws = _workspace(need, x)
    _check(L.fb_layer_norm_grad(pdy, lddy, px, ldx, pm, pr, pw, wtype, R, H, code, dx.data_ptr() if want_dx else None, H,
                                dw.data_ptr() if want_dweight else None, db.data_ptr() if want_dbias else None, pws, need, _raw_stream(dev)))
    return dx, dw, db


def _activation(name: str) -> int:
    if name not in ACTIVATIONS:
        raise ValueError(f"activation must be one of {', '.join(ACTIVATIONS)}")
    return ACTIVATIONS[name]


def fb_affine(x, weight, bias=None, activation: str = "none", residual=None, out_dtype=None, want_preact: bool = False):
    """-> y = activation(x weight^T + bias) + residual, [..., N], or with want_preact (y, preact).

    ``x`` [..., K]; ``weight`` [N, K] of x's type; ``bias`` [N] float32; ``residual`` [..., N] of the output's type;
    ``out_dtype``: x's type (None) or float32; preact, of x's type: what the activation was applied to."""
    L = lib()
    code, act = _type(x, "x"), _activation(activation)
    px, ldx, M, K, dev = _rows(x, "x")
    if weight.dim() != 2:
        raise ValueError("weight must be [N, K]")
    pw, ldw, _, _, _ = _rows(weight, "weight", K, x.dtype, None, dev)
    N = int(weight.shape[0])
    pb = _vector(bias, "bias", N, (torch.float32,), dev)
    out = x.dtype if out_dtype is None else out_dtype
    if out not in (x.dtype, torch.float32):
        raise ValueError("out_dtype must be x's type or float32")
    lead = x.shape[:-1]
    pr, ldr = None, N
    if residual is not None:
        pr, ldr, _, _, _ = _rows(residual, "residual", N, out, lead, dev)
    y = _out(x, (*lead, N), out)
    z = _out(x, (*lead, N), x.dtype) if want_preact else None
    need = int(L.fb_affine_workspace_bytes(px, ldx, pw, ldw, M, N, K, code))
    ws, pws = _workspace(need, x)
    _check(L.fb_affine(px, ldx, pw, ldw, pb, pr, ldr, M, N, K, code, act, y.data_ptr(), N, _types[out],
                       z.data_ptr() if want_preact else None, N, pws, need, _raw_stream(dev)))
    return (y, z) if want_preact else y


def fb_affine_grad(dy, x, weight, activation: str = "none", preact=None, want_dx: bool = True, want_dweight: bool = True,
                   want_dbias: bool = True):
    """-> (dx like x, dweight like weight, dbias [N] float32), None in the place of one that is not wanted.

    ``dy`` [..., N] of x's type or float32; ``preact`` [..., N] of x's type, as fb_affine returned it (needed unless the
    activation is "none").  The gradient of the residual is dy itself."""
    L = lib()
    code, act = _type(x, "x"), _activation(activation)
    px, ldx, M, K, dev = _rows(x, "x")
    if weight.dim() != 2:
        raise ValueError("weight must be [N, K]")
    pw, ldw, _, _, _ = _rows(weight, "weight", K, x.dtype, None, dev)
    N = int(weight.shape[0])
    if dy.dtype not in (x.dtype, torch.float32):
        raise ValueError("dy must be of x's type or float32")
    pdy, lddy, _, _, _ = _rows(dy, "dy", N, None, x.shape[:-1], dev)
    pz, ldz = None, N
    if act:
        if preact is None:
            raise ValueError("preact is needed for this activation")
        pz, ldz, _, _, _ = _rows(preact, "preact", N, x.dtype, x.shape[:-1], dev)
    dx = _out_like(x) if want_dx else None
    dw = _out(x, (N, K), x.dtype) if want_dweight else None
    db = _out(x, (N,), torch.float32) if want_dbias else None
    dtype = _types[dy.dtype]
    need = int(L.fb_affine_grad_workspace_bytes(pdy, lddy, dtype, px, ldx, pw, ldw, M, N, K, code, act))
    ws, pws = _workspace(need, x)
    _check(L.fb_affine_grad(pdy, lddy, dtype, px, ldx, pw, ldw, pz, ldz, M, N, K, code, act, dx.data_ptr() if want_dx else None, K,
                            dw.data_ptr() if want_dweight else None, db.data_ptr() if want_dbias else None, pws, need, _raw_stream(dev)))
    return dx, dw, db


def fb_token_logprobs(logits, tokens, top: int = 0):
    """-> (logprobs, entropy, logz: float32 of the leading shape, top_ids int32 and top_logprobs float32 [..., top]).

    ``logits`` [..., V]; ``tokens`` int32 of the leading shape, negative where a row does not count (its outputs are 0, its
    top_ids -1)."""
    L = lib()
    code = _type(logits, "logits")
    p, ld, R, V, dev = _rows(logits, "logits")
    lead = logits.shape[:-1]
    if tokens.shape != lead:
        raise ValueError("tokens must have the leading shape of logits")
    pt = _vector(tokens, "tokens", R, (torch.int32,), dev)
    lp, ent, z = _floats(3, logits, lead)
    best = _out(logits, (*lead, max(top, 0)), torch.float32)
    ids = _out_like(best, torch.int32)
    need = int(L.fb_token_logprobs_workspace_bytes(R, V, code, top))
    ws, pws = _workspace(need, logits)
    _check(L.fb_token_logprobs(p, ld, pt, R, V, code, top, lp.data_ptr(), ent.data_ptr(), z.data_ptr(), ids.data_ptr(),
                               best.data_ptr(), pws, need, _raw_stream(dev)))
    return lp, ent, z, ids, best


def fb_token_logprobs_grad(logits, tokens, logz, entropy, g_logprobs, g_entropy=None):
    """-> dlogits like logits, from the gradients of logprobs and (optional) entropy and what fb_token_logprobs returned."""
    L = lib()
    code = _type(logits, "logits")
    p, ld, R, V, dev = _rows(logits, "logits")
    if tokens.shape != logits.shape[:-1]:
        raise ValueError("tokens must have the leading shape of logits")
    f = (torch.float32,)
    pt, pz = _vector(tokens, "tokens", R, (torch.int32,), dev), _vector(logz, "logz", R, f, dev)
    pe = _vector(entropy, "entropy", R, f, dev)
    pg, ph = _vector(g_logprobs, "g_logprobs", R, f, dev), _vector(g_entropy, "g_entropy", R, f, dev)
    d = _out_like(logits)
    _check(L.fb_token_logprobs_grad(p, ld, pt, pz, pe, pg, ph, R, V, code, d.data_ptr(), V, _raw_stream(dev)))
    return d
