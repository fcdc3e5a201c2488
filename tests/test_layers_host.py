"""The network-side operators' C entry points without a GPU: every declared symbol is there, malformed arguments come back
as codes with a message, and workspaces are what the calls ask for."""
import ctypes
import os
import re

import pytest

import paper_2112_00709_amd as fb
from paper_2112_00709_amd import layers

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not os.path.exists(fb.LIB_PATH):
        from paper_2112_00709_amd import build
        build.build_library()


def test_library_exports_every_declared_symbol():
    header = open(os.path.join(ROOT, "include", "fb_layers.h")).read()
    header = re.sub(r"/\*.*?\*/", "", header, flags=re.S)
    declared = set(re.findall(r"\b(fb_\w+)\s*\(", header))
    assert declared == set(layers.SYMBOLS)
    for name in declared:
        assert getattr(layers.lib(), name) is not None


def _one():
    return ctypes.c_void_p(4096)          # an address that a refused call does not follow


NORM = dict(x=_one(), ldx=8, weight=None, bias=None, wtype=0, R=4, H=8, type=0, eps=1e-5, y=_one(), ldy=8, mean=None, rstd=None, stream=None)
NORM_GRAD = dict(dy=_one(), lddy=8, x=_one(), ldx=8, mean=_one(), rstd=_one(), weight=None, wtype=0, R=4, H=8, type=0, dx=_one(), lddx=8,
                 dweight=_one(), dbias=None, ws=_one(), ws_bytes=1 << 20, stream=None)
AFFINE = dict(x=_one(), ldx=8, weight=_one(), ldw=8, bias=None, residual=None, ldr=6, M=4, N=6, K=8, type=0, act=0, y=_one(), ldy=6, out_type=0,
              preact=None, ldp=6, ws=_one(), ws_bytes=1 << 20, stream=None)
AFFINE_GRAD = dict(dy=_one(), lddy=6, dy_type=0, x=_one(), ldx=8, weight=_one(), ldw=8, preact=None, ldp=6, M=4, N=6, K=8, type=0, act=0, dx=_one(),
                   lddx=8, dweight=_one(), dbias=_one(), ws=_one(), ws_bytes=1 << 20, stream=None)
TOKENS = dict(logits=_one(), ld=8, tokens=_one(), R=4, V=8, type=0, top=2, logprobs=None, entropy=None, logz=None, top_ids=_one(), top_logprobs=_one(),
              ws=None, ws_bytes=0, stream=None)
TOKENS_GRAD = dict(logits=_one(), ld=8, tokens=_one(), logz=_one(), entropy=_one(), g_logprobs=_one(), g_entropy=_one(), R=4, V=8, type=0,
                   dlogits=_one(), ldd=8, stream=None)
BAD = [("fb_layer_norm", NORM, dict(x=None), dict(y=None), dict(R=-1), dict(R=1 << 31), dict(H=0), dict(H=1 << 31), dict(ldx=7), dict(ldy=7), dict(type=3),
        dict(wtype=1), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf"))),
       ("fb_layer_norm_grad", NORM_GRAD, dict(x=None), dict(dy=None), dict(mean=None), dict(rstd=None), dict(ws=None), dict(ws_bytes=8), dict(lddx=7), dict(lddy=7),
        dict(type=-1)),
       ("fb_affine", AFFINE, dict(x=None), dict(weight=None), dict(y=None), dict(M=-1), dict(N=0), dict(K=0), dict(ldx=7), dict(ldw=7), dict(ldy=5), dict(act=4),
        dict(act=-1), dict(out_type=1), dict(type=5), dict(residual=_one(), ldr=5), dict(preact=_one(), ldp=5), dict(K=1 << 31, ldx=1 << 31, ldw=1 << 31)),
       ("fb_affine_grad", AFFINE_GRAD, dict(dy=None), dict(x=None), dict(weight=None), dict(act=1), dict(dy_type=1), dict(lddy=5), dict(lddx=7), dict(ws=None),
        dict(ws_bytes=8)),
       ("fb_token_logprobs", TOKENS, dict(logits=None), dict(tokens=None), dict(top=-1), dict(top=9), dict(V=100, ld=100, top=65), dict(top_ids=None),
        dict(top_logprobs=None), dict(ld=7), dict(V=0), dict(R=-5), dict(type=7), dict(V=1 << 20, ld=1 << 20)),
       ("fb_token_logprobs_grad", TOKENS_GRAD, dict(logits=None), dict(tokens=None), dict(logz=None), dict(entropy=None), dict(dlogits=None), dict(ldd=7), dict(ld=7))]


@pytest.mark.parametrize("name,good,change", [(b[0], b[1], c) for b in BAD for c in b[2:]])
def test_malformed_arguments_are_codes(name, good, change):
    rc = getattr(layers.lib(), name)(*{**good, **change}.values())
    assert rc == fb.FB_EINVAL
    assert name.encode() in fb.lib().fb_last_error()


def test_sizes_beyond_the_kernels_addresses_are_codes():
    L = layers.lib()
    far = 1 << 27
    for change in [dict(M=65, ldy=far), dict(M=65, residual=_one(), ldr=far), dict(M=65, preact=_one(), ldp=far),
                   dict(M=65, K=(1 << 20) + 1, ldx=1 << 21, ldw=1 << 21), dict(N=1 << 26, ldy=1 << 26)]:
        assert L.fb_affine(*{**AFFINE, **change}.values()) == fb.FB_EUNSUPPORTED
    for change in [dict(lddx=far), dict(K=(1 << 20) + 1, ldx=1 << 21, ldw=1 << 21, lddx=1 << 21)]:
        assert L.fb_affine_grad(*{**AFFINE_GRAD, **change}.values()) == fb.FB_EUNSUPPORTED


def test_workspaces():
    L = layers.lib()
    assert L.fb_layer_norm_grad_workspace_bytes(0, 10) > 0 and L.fb_layer_norm_grad_workspace_bytes(-1, 10) == 0
    assert L.fb_layer_norm_grad_workspace_bytes(1000, 64) % 256 == 0
    assert L.fb_token_logprobs_workspace_bytes(4, 100, 0, 3) == 0                    # one launch, nothing kept
    assert L.fb_token_logprobs_workspace_bytes(1, 1 << 17, 1, 3) > 0
    assert L.fb_token_logprobs_workspace_bytes(1, 1 << 17, 1, 65) == 0
    assert L.fb_affine_grad_workspace_bytes(_one(), 10, 2, _one(), 10, _one(), 10, 10, 10, 10, 1, 0) == 0    # dy of another 16-bit type
    assert L.fb_affine_grad_workspace_bytes(_one(), 10, 0, _one(), 10, _one(), 10, 10, 10, 10, 1, 0) > 0
    assert L.fb_affine_workspace_bytes(_one(), 64, _one(), 64, 999, 64, 64, 1) == 0       # whole pieces, one share of k
    assert L.fb_affine_workspace_bytes(_one(), 65, _one(), 64, 999, 64, 64, 1) >= 999 * 128


def test_no_rows_is_no_work():
    L = layers.lib()
    assert L.fb_layer_norm(*{**NORM, "R": 0, "x": None, "y": None}.values()) == fb.FB_OK
    assert L.fb_affine(*{**AFFINE, "M": 0, "x": None, "y": None}.values()) == fb.FB_OK
    assert L.fb_token_logprobs(*{**TOKENS, "R": 0}.values()) == fb.FB_OK
    assert L.fb_token_logprobs_grad(*{**TOKENS_GRAD, "R": 0}.values()) == fb.FB_OK
