"""C entry points of the block operators without a GPU: malformed arguments come back as codes with a message, and workspaces are what the
calls ask for."""
import ctypes
import os

import pytest

import paper_2112_00709_amd as fb
from paper_2112_00709_amd import layers


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not os.path.exists(fb.LIB_PATH):
        from paper_2112_00709_amd import build
        build.build_library()


def _one():
    return ctypes.c_void_p(4096)          # an address that a refused call does not follow


RESIDUAL = dict(h=_one(), ldh=8, residual=_one(), ldr=8, gate=_one(), ldg=8, scale=0.5, inner=1, inner_weight=_one(), inner_bias=None, outer=2,
                weight=_one(), bias=None, wtype=0, R=4, H=8, type=0, eps=1e-5, s=_one(), lds=8, y=_one(), ldy=8, stats=None, stream=None)
RESIDUAL_GRAD = dict(ds=_one(), ldds=8, dy=_one(), lddy=8, h=_one(), ldh=8, s=_one(), lds=8, stats=_one(), gate=_one(), ldg=8, scale=0.5, inner=1,
                     inner_weight=_one(), inner_bias=None, outer=2, weight=_one(), wtype=0, R=4, H=8, type=0, dh=_one(), lddh=8, dresidual=_one(),
                     lddr=8, dgate=_one(), lddg=8, dinner_weight=_one(), dinner_bias=_one(), dweight=_one(), dbias=_one(), ws=_one(), ws_bytes=1 << 20,
                     stream=None)
GATED = dict(x=_one(), ldx=8, weight=_one(), ldw=8, bias=None, M=4, N=6, K=8, type=0, act=4, y=_one(), ldy=6, preact=_one(), ldp=12, ws=_one(),
             ws_bytes=1 << 20, stream=None)
GATED_GRAD = dict(dy=_one(), lddy=6, x=_one(), ldx=8, weight=_one(), ldw=8, preact=_one(), ldp=12, M=4, N=6, K=8, type=0, act=4, dx=_one(), lddx=8,
                  dweight=_one(), dbias=_one(), ws=_one(), ws_bytes=1 << 20, stream=None)
SCORES = dict(x=_one(), ldx=8, weight=_one(), ldw=8, bias=None, tokens=_one(), M=4, V=6, K=8, type=0, logprobs=_one(), entropy=_one(), logz=_one(),
              ws=_one(), ws_bytes=1 << 20, stream=None)
SCORES_GRAD = dict(x=_one(), ldx=8, weight=_one(), ldw=8, bias=None, tokens=_one(), logz=_one(), entropy=_one(), g_logprobs=_one(), g_entropy=_one(),
                   M=4, V=6, K=8, type=0, dx=_one(), lddx=8, dweight=_one(), dbias=_one(), ws=_one(), ws_bytes=1 << 20, stream=None)
SIZES = [dict(K=0), dict(K=1 << 28, ldx=1 << 28, ldw=1 << 28), dict(M=-1), dict(M=1 << 31), dict(ldx=7), dict(ldw=7), dict(type=3), dict(type=-1),
         dict(x=None), dict(weight=None)]
BAD = [("fb_residual_norm", RESIDUAL, dict(h=None), dict(s=None), dict(y=None), dict(R=-1), dict(R=1 << 31), dict(H=0), dict(ldh=7), dict(ldr=7), dict(ldg=7), dict(lds=7),
        dict(ldy=7), dict(type=3), dict(wtype=1), dict(inner=3), dict(outer=-1), dict(inner=0), dict(outer=0), dict(eps=-1.0), dict(eps=float("nan")),
        dict(eps=float("inf")), dict(scale=float("inf")), dict(scale=float("nan"))),
       ("fb_residual_norm_grad", RESIDUAL_GRAD, dict(dy=None), dict(s=None), dict(h=None), dict(stats=None), dict(ldds=7), dict(lddy=7), dict(ldh=7), dict(lds=7),
        dict(ldg=7), dict(lddh=7), dict(lddr=7), dict(lddg=7), dict(ws=None), dict(ws_bytes=8), dict(gate=None), dict(inner=0, inner_weight=None),
        dict(outer=0, weight=None), dict(outer=0, weight=None, dweight=None, dbias=None, ds=None), dict(type=9), dict(wtype=2), dict(scale=float("nan"))),
       ("fb_gated_affine", GATED, *SIZES, dict(N=0), dict(N=1 << 27, ldy=1 << 27, ldp=1 << 28), dict(y=None), dict(ldy=5), dict(ldp=11), dict(act=5), dict(act=-1)),
       ("fb_gated_affine_grad", GATED_GRAD, *SIZES, dict(N=0), dict(dy=None), dict(preact=None), dict(lddy=5), dict(ldp=11), dict(lddx=7), dict(act=5), dict(ws=None),
        dict(ws_bytes=8)),
       ("fb_affine_logprobs", SCORES, *SIZES, dict(V=0), dict(V=1 << 28), dict(tokens=None), dict(ws=None), dict(ws_bytes=8)),
       ("fb_affine_logprobs_grad", SCORES_GRAD, *SIZES, dict(V=0), dict(V=1 << 28), dict(tokens=None), dict(logz=None), dict(entropy=None), dict(lddx=7), dict(ws=None),
        dict(ws_bytes=8))]


@pytest.mark.parametrize("name,good,change", [(b[0], b[1], c) for b in BAD for c in b[2:]])
def test_malformed_arguments_are_codes(name, good, change):
    rc = getattr(layers.lib(), name)(*{**good, **change}.values())
    assert rc == fb.FB_EINVAL
    assert name.encode() in fb.lib().fb_last_error()


def test_sizes_beyond_the_kernels_are_codes():
    L = layers.lib()
    far, long = 1 << 27, dict(K=(1 << 20) + 1, ldx=1 << 21, ldw=1 << 21)
    assert L.fb_residual_norm(*{**RESIDUAL, **{k: 8193 for k in ("H", "ldh", "ldr", "ldg", "lds", "ldy")}}.values()) == fb.FB_EUNSUPPORTED
    assert L.fb_residual_norm_grad(*{**RESIDUAL_GRAD, **{k: 8193 for k in ("H", "ldds", "lddy", "ldh", "lds", "ldg", "lddh", "lddr", "lddg")}}.values()) == fb.FB_EUNSUPPORTED
    for change in [dict(M=65, ldy=far), dict(M=65, ldp=far), dict(M=65, **long), dict(N=1 << 25, ldy=1 << 25, ldp=1 << 26)]:
        assert L.fb_gated_affine(*{**GATED, **change}.values()) == fb.FB_EUNSUPPORTED
    for change in [dict(lddx=far), dict(lddx=1 << 21, **long), dict(N=(1 << 19) + 1, lddy=1 << 20, ldp=1 << 21)]:
        assert L.fb_gated_affine_grad(*{**GATED_GRAD, **change}.values()) == fb.FB_EUNSUPPORTED
    assert L.fb_affine_logprobs(*{**SCORES, **long}.values()) == fb.FB_EUNSUPPORTED
    for change in [dict(lddx=far), dict(lddx=1 << 21, **long)]:
        assert L.fb_affine_logprobs_grad(*{**SCORES_GRAD, **change}.values()) == fb.FB_EUNSUPPORTED


def test_workspaces():
    L = layers.lib()
    p = _one()
    assert L.fb_residual_norm_grad_workspace_bytes(0, 10) > 0 and L.fb_residual_norm_grad_workspace_bytes(9, 8193) == 0
    assert L.fb_gated_affine_workspace_bytes(p, 64, p, 64, 4, 4096, 64, 1) == 0                      # few rows
    assert L.fb_gated_affine_workspace_bytes(p, 64, p, 64, 44160, 2048, 64, 1) == 0                  # whole pieces, one share of k
    assert L.fb_gated_affine_workspace_bytes(p, 65, p, 64, 44160, 2048, 64, 1) >= 44160 * 128
    assert L.fb_gated_affine_grad_workspace_bytes(p, 64, p, 64, 1000, 300, 64, 1) >= 1000 * 600 * 2
    assert L.fb_gated_affine_grad_workspace_bytes(p, 64, p, 64, 1000, 0, 64, 1) == 0
    for M in (0, 1, 64, 65, 4095):
        for type in (0, 1, 2):
            assert L.fb_affine_logprobs_workspace_bytes(p, 64, p, 64, M, 128000, 64, type) > 0
            assert L.fb_affine_logprobs_grad_workspace_bytes(p, 64, p, 64, M, 128000, 64, type) > 0
    # the logits of 4095 x 128000 would be 1 GB: forward none of them, in the gradient half at a time
    assert L.fb_affine_logprobs_workspace_bytes(p, 2048, p, 2048, 4095, 128000, 2048, 1) < 64 << 20
    assert L.fb_affine_logprobs_grad_workspace_bytes(p, 2048, p, 2048, 4095, 128000, 2048, 1) < 1 << 30
    assert L.fb_affine_logprobs_grad_workspace_bytes(p, 64, p, 64, 4, 128000, 64, 3) == 0


def test_no_rows_is_no_work():
    L = layers.lib()
    assert L.fb_residual_norm(*{**RESIDUAL, "R": 0, "h": None, "s": None, "y": None}.values()) == fb.FB_OK
    assert L.fb_gated_affine(*{**GATED, "M": 0, "x": None, "y": None}.values()) == fb.FB_OK
    assert L.fb_affine_logprobs(*{**SCORES, "M": 0, "x": None, "tokens": None}.values()) == fb.FB_OK
    assert L.fb_affine_logprobs_grad(*{**SCORES_GRAD, "M": 0, "dx": None, "dweight": None, "dbias": None}.values()) == fb.FB_OK
