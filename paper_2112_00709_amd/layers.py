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

from . import FBError, _check, _new, lib as _base_lib  # noqa: F401  (FBError: what a failing call raises)

F32, BF16, F16 = 0, 1, 2
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
TOP_MAX = 64

# every symbol include/fb_layers.h declares
SYMBOLS = ["fb_layer_norm", "fb_layer_norm_grad_workspace_bytes", "fb_layer_norm_grad", "fb_affine_workspace_bytes", "fb_affine",
           "fb_affine_grad_workspace_bytes", "fb_affine_grad", "fb_token_logprobs_workspace_bytes", "fb_token_logprobs",
           "fb_token_logprobs_grad"]

_lib = None
_types = None


def lib() -> ctypes.CDLL:
    """The built library with these calls' signatures (fails loudly when it has not been built)."""
    global _lib, _types
    if _lib is None:
        L = _base_lib()
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
        import torch
        _types = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}
        _lib = L
    return _lib


def _torch():
    import torch
    return torch


def _type(t, what: str) -> int:
    lib()
    code = _types.get(t.dtype)
    if code is None:
        raise ValueError(f"{what} must be float32, bfloat16 or float16")
    return code


def _rows(t, what: str, width: Optional[int] = None, dtype=None, lead=None):
    """-> (address, row distance, rows, width) of [..., width] as rows."""
    torch = _torch()
    if not t.is_cuda or t.dim() < 1:
        raise ValueError(f"{what} must be a CUDA tensor of at least one dimension")
    if t.device.index != torch.cuda.current_device():
        raise ValueError(f"{what} must lie on the current device")
    if width is not None and t.shape[-1] != width:
        raise ValueError(f"{what} must have rows of {width} elements")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{what} must be {dtype}")
    if lead is not None and t.shape[:-1] != lead:
        raise ValueError(f"{what} must have the same rows as the first argument")
    w = t.shape[-1]
    n = t.numel() // w if w else 0
    if t.is_contiguous():
        return t.data_ptr(), w, n, w
    if w > 1 and t.stride(-1) != 1:
        raise ValueError(f"the elements of a row of {what} must be contiguous")
    ld = 0                                       # the leading dimensions have to be one walk over the rows
    for size, step in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if size == 1:
            continue
        if ld == 0:
            ld, seen = step, size
        elif step != ld * seen:
            raise ValueError(f"the rows of {what} must lie at one distance")
        else:
            seen *= size
    if ld == 0:
        ld = w
    if ld < w and n > 1:
        raise ValueError(f"the rows of {what} must not overlap")
    return t.data_ptr(), ld, n, w


def _vector(t, what: str, n: int, dtypes):
    if t is None:
        return None
    if not (t.is_cuda and t.is_contiguous() and t.numel() == n and t.dtype in dtypes):
        raise ValueError(f"{what} must be a contiguous CUDA tensor of {n} elements of {' or '.join(str(d) for d in dtypes)}")
    if t.device.index != _torch().cuda.current_device():
        raise ValueError(f"{what} must lie on the current device")
    return t.data_ptr()


def _stream():
    return _torch().cuda.current_stream().cuda_stream


def _workspace(n: int, device):
    if n == 0:
        return None, None
    ws = _new((n,), _torch().uint8, device)
    return ws, ws.data_ptr()


def fb_layer_norm(x, weight=None, bias=None, eps: float = 1e-5, want_stats: bool = False):
    """-> y like x, or with want_stats (y, mean, rstd), the latter float32 of x's leading shape.

    ``x`` [..., H]; ``weight``, ``bias`` [H], float32 or of x's type (both of one)."""
    torch = _torch()
    L = lib()
    code = _type(x, "x")
    px, ldx, R, H = _rows(x, "x")
    wt = weight if weight is not None else bias
    wtype = F32 if wt is None else _type(wt, "weight")
    if weight is not None and bias is not None and weight.dtype != bias.dtype:
        raise ValueError("weight and bias must have one type")
    pw, pb = _vector(weight, "weight", H, (torch.float32, x.dtype)), _vector(bias, "bias", H, (torch.float32, x.dtype))
    y = _new(x.shape, x.dtype, x.device)
    mean = rstd = pm = pr = None
    if want_stats:
        mean, rstd = _new(x.shape[:-1], torch.float32, x.device), _new(x.shape[:-1], torch.float32, x.device)
        pm, pr = mean.data_ptr(), rstd.data_ptr()
    _check(L.fb_layer_norm(px, ldx, pw, pb, wtype, R, H, code, eps, y.data_ptr(), H, pm, pr, _stream()))
    return (y, mean, rstd) if want_stats else y


def fb_layer_norm_grad(dy, x, mean, rstd, weight=None, want_dx: bool = True, want_dweight: bool = True, want_dbias: bool = True):
    """-> (dx like x, dweight [H] float32, dbias [H] float32), None in the place of one that is not wanted.

    ``dy`` like x; ``mean``, ``rstd``: as fb_layer_norm returned them."""
    torch = _torch()
    L = lib()
    code = _type(x, "x")
    px, ldx, R, H = _rows(x, "x")
    pdy, lddy, _, _ = _rows(dy, "dy", H, x.dtype, x.shape[:-1])
    pm, pr = _vector(mean, "mean", R, (torch.float32,)), _vector(rstd, "rstd", R, (torch.float32,))
    wtype = F32 if weight is None else _type(weight, "weight")
    pw = _vector(weight, "weight", H, (torch.float32, x.dtype))
    dx = _new(x.shape, x.dtype, x.device) if want_dx else None
    dw = _new((H,), torch.float32, x.device) if want_dweight else None
    db = _new((H,), torch.float32, x.device) if want_dbias else None
    need = int(L.fb_layer_norm_grad_workspace_bytes(R, H)) if want_dweight or want_dbias else 0
    ws, pws = _workspace(need, x.device)
    _check(L.fb_layer_norm_grad(pdy, lddy, px, ldx, pm, pr, pw, wtype, R, H, code, dx.data_ptr() if want_dx else None, H,
                                dw.data_ptr() if want_dweight else None, db.data_ptr() if want_dbias else None, pws, need, _stream()))
    return dx, dw, db


def _activation(name: str) -> int:
    if name not in ACTIVATIONS:
        raise ValueError(f"activation must be one of {', '.join(ACTIVATIONS)}")
    return ACTIVATIONS[name]


def fb_affine(x, weight, bias=None, activation: str = "none", residual=None, out_dtype=None, want_preact: bool = False):
    """-> y = activation(x weight^T + bias) + residual, [..., N], or with want_preact (y, preact).

    ``x`` [..., K]; ``weight`` [N, K] of x's type; ``bias`` [N] float32; ``residual`` [..., N] of the output's type;
    ``out_dtype``: x's type (None) or float32; preact, of x's type: what the activation was applied to."""
    torch = _torch()
    L = lib()
    code, act = _type(x, "x"), _activation(activation)
    px, ldx, M, K = _rows(x, "x")
    if weight.dim() != 2:
        raise ValueError("weight must be [N, K]")
    pw, ldw, N, _ = _rows(weight, "weight", K, x.dtype)
    N = int(weight.shape[0])
    pb = _vector(bias, "bias", N, (torch.float32,))
    out = x.dtype if out_dtype is None else out_dtype
    if out not in (x.dtype, torch.float32):
        raise ValueError("out_dtype must be x's type or float32")
    lead = x.shape[:-1]
    pr, ldr = None, N
    if residual is not None:
        pr, ldr, _, _ = _rows(residual, "residual", N, out, lead)
    y = _new((*lead, N), out, x.device)
    z = _new((*lead, N), x.dtype, x.device) if want_preact else None
    need = int(L.fb_affine_workspace_bytes(px, ldx, pw, ldw, M, N, K, code))
    ws, pws = _workspace(need, x.device)
    _check(L.fb_affine(px, ldx, pw, ldw, pb, pr, ldr, M, N, K, code, act, y.data_ptr(), N, _types[out],
                       z.data_ptr() if want_preact else None, N, pws, need, _stream()))
    return (y, z) if want_preact else y


def fb_affine_grad(dy, x, weight, activation: str = "none", preact=None, want_dx: bool = True, want_dweight: bool = True,
                   want_dbias: bool = True):
    """-> (dx like x, dweight like weight, dbias [N] float32), None in the place of one that is not wanted.

    ``dy`` [..., N] of x's type or float32; ``preact`` [..., N] of x's type, as fb_affine returned it (needed unless the
    activation is "none").  The gradient of the residual is dy itself."""
    torch = _torch()
    L = lib()
    code, act = _type(x, "x"), _activation(activation)
    px, ldx, M, K = _rows(x, "x")
    if weight.dim() != 2:
        raise ValueError("weight must be [N, K]")
    pw, ldw, _, _ = _rows(weight, "weight", K, x.dtype)
    N = int(weight.shape[0])
    if dy.dtype not in (x.dtype, torch.float32):
        raise ValueError("dy must be of x's type or float32")
    pdy, lddy, _, _ = _rows(dy, "dy", N, None, x.shape[:-1])
    pz, ldz = None, N
    if act:
        if preact is None:
            raise ValueError("preact is needed for this activation")
        pz, ldz, _, _ = _rows(preact, "preact", N, x.dtype, x.shape[:-1])
    dx = _new(x.shape, x.dtype, x.device) if want_dx else None
    dw = _new((N, K), x.dtype, x.device) if want_dweight else None
    db = _new((N,), torch.float32, x.device) if want_dbias else None
    dtype = _types[dy.dtype]
    need = int(L.fb_affine_grad_workspace_bytes(pdy, lddy, dtype, px, ldx, pw, ldw, M, N, K, code, act))
    ws, pws = _workspace(need, x.device)
    _check(L.fb_affine_grad(pdy, lddy, dtype, px, ldx, pw, ldw, pz, ldz, M, N, K, code, act, dx.data_ptr() if want_dx else None, K,
                            dw.data_ptr() if want_dweight else None, db.data_ptr() if want_dbias else None, pws, need, _stream()))
    return dx, dw, db


def fb_token_logprobs(logits, tokens, top: int = 0):
    """-> (logprobs, entropy, logz: float32 of the leading shape, top_ids int32 and top_logprobs float32 [..., top]).

    ``logits`` [..., V]; ``tokens`` int32 of the leading shape, negative where a row does not count (its outputs are 0, its
    top_ids -1)."""
    torch = _torch()
    L = lib()
    code = _type(logits, "logits")
    p, ld, R, V = _rows(logits, "logits")
    lead = logits.shape[:-1]
    if tokens.shape != lead:
        raise ValueError("tokens must have the leading shape of logits")
    pt = _vector(tokens, "tokens", R, (torch.int32,))
    dev = logits.device
    lp, ent, z = (_new(lead, torch.float32, dev) for _ in range(3))
    ids, best = _new((*lead, top), torch.int32, dev), _new((*lead, top), torch.float32, dev)
    need = int(L.fb_token_logprobs_workspace_bytes(R, V, code, top))
    ws, pws = _workspace(need, dev)
    _check(L.fb_token_logprobs(p, ld, pt, R, V, code, top, lp.data_ptr(), ent.data_ptr(), z.data_ptr(), ids.data_ptr(),
                               best.data_ptr(), pws, need, _stream()))
    return lp, ent, z, ids, best


def fb_token_logprobs_grad(logits, tokens, logz, entropy, g_logprobs, g_entropy=None):
    """-> dlogits like logits, from the gradients of logprobs and (optional) entropy and what fb_token_logprobs returned."""
    torch = _torch()
    L = lib()
    code = _type(logits, "logits")
    p, ld, R, V = _rows(logits, "logits")
    if tokens.shape != logits.shape[:-1]:
        raise ValueError("tokens must have the leading shape of logits")
    f = (torch.float32,)
    pt, pz = _vector(tokens, "tokens", R, (torch.int32,)), _vector(logz, "logz", R, f)
    pe = _vector(entropy, "entropy", R, f)
    pg, ph = _vector(g_logprobs, "g_logprobs", R, f), _vector(g_entropy, "g_entropy", R, f)
    d = _new(logits.shape, logits.dtype, logits.device)
    _check(L.fb_token_logprobs_grad(p, ld, pt, pz, pe, pg, ph, R, V, code, d.data_ptr(), V, _stream()))
    return d
