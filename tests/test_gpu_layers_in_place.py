"""The last layers' C entry points where an output lies on an input, as the header allows, against the same call with an output of
its own, bit by bit; narrow outputs; and outputs so large that they are stored past the caches."""
from __future__ import annotations

import math

import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
H_OF = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
CODE = {"float32": 0, "bfloat16": 1, "float16": 2}


@pytest.fixture(scope="module")
def fl():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_2112_00709_amd as base
    from paper_2112_00709_amd import layers
    layers.lib()
    base.POISON_NEW_BUFFERS = True
    return layers


def rows(n, width, dtype, seed, scale=1.0):
    import torch
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((n, width), generator=g) * scale).to(getattr(torch, dtype)).cuda()


def ok(fl, rc):
    import torch
    fl._check(rc)
    torch.cuda.synchronize()


def stream():
    import torch
    return torch.cuda.current_stream().cuda_stream


def address(t):
    return None if t is None else t.data_ptr()


# rows of one, four and sixteen waves, and those that are read again
@pytest.mark.parametrize("R,H", [(1, 8), (9001, 300), (700, 1500), (1200, 5000), (40, 20000), (3, 16385)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_layer_norm(fl, R, H, dtype):
    import torch
    x, dy, w, b = rows(R, H, dtype, 1), rows(R, H, dtype, 2), 1 + rows(1, H, "float32", 3)[0], rows(1, H, "float32", 4)[0]
    y, mean, rstd = fl.fb_layer_norm(x, w, b, want_stats=True)
    L, on = fl.lib(), x.clone()
    m2, r2 = torch.empty_like(mean), torch.empty_like(rstd)
    ok(fl, L.fb_layer_norm(address(on), H, address(w), address(b), 0, R, H, CODE[dtype], 1e-5, address(on), H, address(m2), address(r2), stream()))
    assert torch.equal(on, y) and torch.equal(m2, mean) and torch.equal(r2, rstd)
    want = fl.fb_layer_norm_grad(dy, x, mean, rstd, w)
    need = L.fb_layer_norm_grad_workspace_bytes(R, H)
    for over in ("dy", "x"):
        ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
        gy, gx, dw, db = dy.clone(), x.clone(), torch.empty_like(w), torch.empty_like(w)
        dx = gy if over == "dy" else gx
        ok(fl, L.fb_layer_norm_grad(address(gy), H, address(gx), H, address(mean), address(rstd), address(w), 0, R, H, CODE[dtype], address(dx), H,
                                    address(dw), address(db), address(ws), need, stream()))
        assert torch.equal(dx, want[0]) and torch.equal(dw, want[1]) and torch.equal(db, want[2])


# few rows, one and more tiles, ragged edges, joined shares of k (N below 4 among them)
@pytest.mark.parametrize("M,N,K", [(5, 70, 40), (64, 513, 40), (300, 3, 70), (300, 1111, 777), (70, 130, 4000), (2000, 520, 264)])
@pytest.mark.parametrize("dtype,out", [("float32", "float32"), ("bfloat16", "bfloat16"), ("float16", "float32")])
@pytest.mark.parametrize("activation", ["none", "gelu"])
def test_affine_onto_its_residual(fl, M, N, K, dtype, out, activation):
    import torch
    x, w, b, r = rows(M, K, dtype, 1), rows(N, K, dtype, 2, K ** -0.5), rows(1, N, "float32", 3)[0], rows(M, N, out, 4)
    want = fl.fb_affine(x, w, b, activation=activation, residual=r, out_dtype=getattr(torch, out))
    L = fl.lib()
    need = L.fb_affine_workspace_bytes(address(x), K, address(w), K, M, N, K, CODE[dtype])
    ws = torch.full((max(need, 1),), 255, dtype=torch.uint8, device="cuda")
    ok(fl, L.fb_affine(address(x), K, address(w), K, address(b), address(r), N, M, N, K, CODE[dtype], fl.ACTIVATIONS[activation], address(r), N,
                       CODE[out], None, N, address(ws), need, stream()))
    assert torch.equal(r, want)


@pytest.mark.parametrize("R,V", [(1000, 84), (37, 700), (9, 1500), (3, 70001)])
@pytest.mark.parametrize("dtype", ["float32", "float16"])
def test_token_gradient_onto_the_logits(fl, R, V, dtype):
    import torch
    x, g, h = rows(R, V, dtype, 1, 3.0), rows(1, R, "float32", 2)[0], rows(1, R, "float32", 3)[0]
    tokens = (torch.arange(R, dtype=torch.int32, device="cuda") * 7) % V
    tokens[1] = -1
    _, ent, z, _, _ = fl.fb_token_logprobs(x, tokens)
    want = fl.fb_token_logprobs_grad(x, tokens, z, ent, g, h)
    ok(fl, fl.lib().fb_token_logprobs_grad(address(x), V, address(tokens), address(z), address(ent), address(g), address(h), R, V, CODE[dtype],
                                           address(x), V, stream()))
    assert torch.equal(x, want)


def held(y, z, x, w, b, r, out):
    """gelu(x w^T + b) + r and what it was applied to, in the bounds of a sum of K products (300 + K / 16 roundings behind one
    another of at most 2 u each), of the activation (slope 1.13, its own 16 u) and of one rounding of the result."""
    import torch
    x, w, b, r, K = x.double().cpu(), w.double().cpu(), b.double().cpu(), r.double().cpu(), x.shape[1]
    want_z = x @ w.t() + b
    e = 2 * (300 + K / 16) * U * (x.abs() @ w.t().abs() + b.abs()) + 1e-37
    want = 0.5 * want_z * (1 + torch.erf(want_z / math.sqrt(2))) + r
    assert ((z.double().cpu() - want_z).abs() <= e + H_OF["float16"] * want_z.abs() * 1.01 + 2.0 ** -24).all()
    tol = 1.13 * e + 16 * U * (1 + want_z.abs()) + 2 * U * want.abs() + H_OF[out] * want.abs() * 1.01 + 2.0 ** -24
    assert ((y.double().cpu() - want).abs() <= tol).all()


@pytest.mark.parametrize("out", ["float16", "float32"])
@pytest.mark.parametrize("M,N,K", [(66, 1, 40), (300, 2, 70), (1000, 3, 2000), (65, 3, 8)])
def test_narrow_outputs_with_everything(fl, M, N, K, out):
    import torch
    x, w, b, r = rows(M, K, "float16", 1), rows(N, K, "float16", 2, K ** -0.5), rows(1, N, "float32", 3)[0], rows(M, N, out, 4)
    y, z = fl.fb_affine(x, w, b, activation="gelu", residual=r, out_dtype=getattr(torch, out), want_preact=True)
    held(y, z, x, w, b, r, out)


@pytest.mark.parametrize("M,N,out", [(21001, 3203, "float16"), (12001, 2803, "float32")])
def test_large_outputs_with_everything(fl, M, N, out):
    """128 MB and more, an odd width: activation, residual, preact."""
    import torch
    K = 72
    x, w, b, r = rows(M, K, "float16", 1), rows(N, K, "float16", 2, K ** -0.5), rows(1, N, "float32", 3)[0], rows(M, N, out, 4)
    y, z = fl.fb_affine(x, w, b, activation="gelu", residual=r, out_dtype=getattr(torch, out), want_preact=True)
    some = torch.cat([torch.arange(0, M, 97), torch.arange(M - 20, M)]).cuda()
    held(y[some], z[some], x[some], w, b, r[some], out)


def test_large_single_precision_outputs(fl):
    import torch
    M, N, K = 12001, 2803, 72
    x, w, b = rows(M, K, "bfloat16", 1), rows(N, K, "bfloat16", 2, K ** -0.5), rows(1, N, "float32", 3)[0]
    y = fl.fb_affine(x, w, b, out_dtype=torch.float32)
    some = torch.cat([torch.arange(0, M, 97), torch.arange(M - 20, M)]).cuda()
    xd, wd = x[some].double().cpu(), w.double().cpu()
    size = xd.abs() @ wd.abs().t() + b.double().cpu().abs()
    assert ((y[some].double().cpu() - (xd @ wd.t() + b.double().cpu())).abs() <= 2 * (300 + K / 16) * U * size).all()


@pytest.mark.parametrize("R,V,dtype", [(2101, 32001, "bfloat16"), (70000, 511, "float32")])
def test_large_token_gradients(fl, R, V, dtype):
    """The rows of a gradient of 128 MB and more are those of the same rows alone."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = (3 * torch.randn((R, V), generator=gen, device="cuda")).to(getattr(torch, dtype))
    g, h = torch.randn(R, generator=gen, device="cuda"), torch.randn(R, generator=gen, device="cuda")
    tokens = torch.arange(R, dtype=torch.int32, device="cuda") % V
    _, ent, z, _, _ = fl.fb_token_logprobs(x, tokens)
    got = fl.fb_token_logprobs_grad(x, tokens, z, ent, g, h)
    some = torch.cat([torch.arange(0, R, 61), torch.arange(R - 9, R)]).cuda()
    few = fl.fb_token_logprobs_grad(*(t[some].contiguous() for t in (x, tokens, z, ent, g, h)))
    assert torch.equal(got[some], few)
