"""Affine layer (bias, activation, residual) and its gradient on the GPU against the definition in 64 bits.

Tolerances.  u = 2^-24, h the type's roundoff.  Products of two 16-bit numbers are exact in single precision; a sum of K of them
is formed with at most n = 300 + K / 16 roundings one after the other (matrix instructions that take 2 or more k at a time, sets
of sums closed from time to time, shares of k and waves joined), each of at most 2 u of what is summed (the instruction may
truncate): e = 2 n u sum |a b|.  Activations have slopes of at most 1.13 and their functions errors of 16 u (1 + |z|).  The
result is rounded once: h.  dz, where it is rounded before the products, adds h of every term's size."""
from __future__ import annotations

import math

import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
H_OF = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
TINY = {"float32": 1e-37, "bfloat16": 1e-37, "float16": 2.0 ** -24}


@pytest.fixture(scope="module")
def fl():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_2112_00709_amd as base
    from paper_2112_00709_amd import layers
    layers.lib()
    base.POISON_NEW_BUFFERS = True
    return layers


def rows(n, width, dtype, gap, seed, scale=1.0):
    """Rows of a wider tensor; what lies between them is NaN."""
    import torch
    g = torch.Generator().manual_seed(seed)
    x = torch.full((n, width + gap), math.nan)
    x[:, :width] = torch.randn((n, width), generator=g) * scale
    return x.to(getattr(torch, dtype)).cuda()[:, :width]


def act(z, name):
    import torch
    if name == "relu":
        return z.clamp_min(0)
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z / math.sqrt(2)))
    if name == "silu":
        return z * torch.sigmoid(z)
    return z


def slope(z, name):
    import torch
    if name == "relu":
        return (z > 0).double()
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z / math.sqrt(2))) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "silu":
        s = torch.sigmoid(z)
        return s + z * s * (1 - s)
    return torch.ones_like(z)


def d(t):
    return t.double().cpu()


def check_forward(fl, M, N, K, dtype, gap, activation, with_bias, with_residual, out, preact, seed=0):
    import torch
    x, w = rows(M, K, dtype, gap, seed + 1), rows(N, K, dtype, gap and 8, seed + 2, K ** -0.5)
    g = torch.Generator().manual_seed(seed + 3)
    b = torch.randn(N, generator=g).cuda() if with_bias else None
    odt = dtype if out == "same" else "float32"
    r = rows(M, N, odt, gap, seed + 4) if with_residual else None
    got = fl.fb_affine(x, w, b, activation=activation, residual=r, out_dtype=None if out == "same" else torch.float32, want_preact=preact)
    y, z = got if preact else (got, None)
    want_z = d(x) @ d(w).t() + (d(b) if with_bias else 0)
    size = d(x).abs() @ d(w).abs().t() + (d(b).abs() if with_bias else 0)
    e = 2 * (300 + K / 16) * U * size + 1e-37
    want = act(want_z, activation) + (d(r) if with_residual else 0)
    tol = 1.13 * e + 16 * U * (1 + want_z.abs()) + 2 * U * want.abs() + H_OF[odt] * want.abs() * 1.01 + TINY[odt]
    assert y.shape == (M, N) and y.dtype == getattr(torch, odt)
    bad = ~((d(y) - want).abs() <= tol)
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist(), d(y)[bad][:4], want[bad][:4])
    if preact:
        assert ((d(z) - want_z).abs() <= e + H_OF[dtype] * want_z.abs() * 1.01 + TINY[dtype]).all() and z.dtype == x.dtype


SIZES = [(1, 1, 1), (1, 2, 3), (1, 84, 512), (1, 2048, 2048), (2, 17, 33), (3, 1000, 1001), (7, 130, 64), (16, 256, 4096), (17, 300, 72), (33, 64, 96),
         (63, 1000, 520), (64, 513, 40), (65, 257, 129), (127, 129, 31), (128, 128, 64), (200, 84, 1024), (255, 250, 255), (256, 256, 256),
         (257, 264, 200), (300, 3000, 128), (1000, 40, 2000), (513, 1111, 777), (2048, 512, 1024), (1500, 1400, 520)]


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("dtype,gap", [("float32", 0), ("bfloat16", 0), ("float16", 3), ("bfloat16", 8)])
def test_forward(fl, M, N, K, dtype, gap):
    k = (M + N + K) % 4
    for v, (activation, with_bias, with_residual, out, preact) in enumerate([
            ("none", False, False, "same", False), ("relu", True, True, "same", True), ("gelu", True, False, "f32", True), ("silu", True, True, "f32", False)]):
        if v == k or v == (k + 1) % 4:
            check_forward(fl, M, N, K, dtype, gap, activation, with_bias, with_residual, out, preact, seed=M + v)


@pytest.mark.parametrize("activation", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("M,N,K", [(5, 70, 40), (260, 264, 136)])
def test_every_epilogue(fl, activation, dtype, M, N, K):
    for with_bias in (False, True):
        for with_residual in (False, True):
            for out in ("same", "f32"):
                for preact in (False, True):
                    check_forward(fl, M, N, K, dtype, 0, activation, with_bias, with_residual, out, preact)


def check_grad(fl, M, N, K, dtype, gap, activation, dy_type, seed=0):
    import torch
    x, w = rows(M, K, dtype, gap, seed + 1), rows(N, K, dtype, gap, seed + 2, K ** -0.5)
    dyt = dtype if dy_type == "same" else "float32"
    dy = rows(M, N, dyt, gap, seed + 3, 0.3)
    z = rows(M, N, dtype, gap, seed + 4, 1.5) if activation != "none" else None
    dx, dw, db = fl.fb_affine_grad(dy, x, w, activation=activation, preact=z)
    g = d(dy) * (slope(d(z), activation) if z is not None else 1)
    h = H_OF[dtype]
    hz = 0.0 if activation == "none" and dyt == dtype else h
    eg = g.abs() * (hz * 1.01 + 4 * U) + 16 * U * d(dy).abs() + (TINY[dtype] if hz else 0)      # error of a dz as the products see it
    want = g @ d(w)
    tol = 2 * (300 + N / 16) * U * (g.abs() @ d(w).abs()) + eg @ d(w).abs()
    assert ((d(dx) - want).abs() <= tol * 1.01 + h * want.abs() * 1.01 + TINY[dtype]).all()
    want = g.t() @ d(x)
    tol = 2 * (300 + M / 16) * U * (g.abs().t() @ d(x).abs()) + eg.t() @ d(x).abs()
    bad = ~((d(dw) - want).abs() <= tol * 1.01 + h * want.abs() * 1.01 + TINY[dtype])
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist(), d(dw)[bad][:4], want[bad][:4])
    tol = (300 + M / 16) * U * g.abs().sum(0) + (g.abs() * 4 * U + 16 * U * d(dy).abs()).sum(0)
    assert ((d(db) - g.sum(0)).abs() <= tol + 1e-37).all()
    assert dx.dtype == x.dtype and dw.dtype == w.dtype and db.dtype == torch.float32


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("dtype,gap", [("float32", 1), ("bfloat16", 0), ("float16", 0), ("bfloat16", 5)])
def test_gradient(fl, M, N, K, dtype, gap):
    k = M + N + K
    check_grad(fl, M, N, K, dtype, gap, ["none", "relu", "gelu", "silu"][k % 4], ["same", "f32"][k // 4 % 2], seed=k)
    check_grad(fl, M, N, K, dtype, gap, "none" if k % 4 else "gelu", "same", seed=k + 9)


@pytest.mark.parametrize("activation", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("dy_type", ["same", "f32"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_every_slope(fl, activation, dy_type, dtype):
    check_grad(fl, 140, 72, 48, dtype, 0, activation, dy_type)
    check_grad(fl, 9, 51, 30, dtype, 2, activation, dy_type)


def test_parts_of_the_gradient(fl):
    """What is left out leaves the rest as it is; a second call gives the same bits."""
    import torch
    x, w, dy, z = rows(3000, 200, "bfloat16", 0, 1), rows(300, 200, "bfloat16", 0, 2), rows(3000, 300, "bfloat16", 0, 3), rows(3000, 300, "bfloat16", 0, 4)
    full = fl.fb_affine_grad(dy, x, w, activation="silu", preact=z)
    for want in [(True, False, False), (False, True, False), (False, False, True), (True, False, True)]:
        got = fl.fb_affine_grad(dy, x, w, activation="silu", preact=z, want_dx=want[0], want_dweight=want[1], want_dbias=want[2])
        for a, b, asked in zip(got, full, want):
            assert (a is None) == (not asked)
            assert not asked or torch.equal(a, b)


def test_gradient_against_differences(fl):
    import torch
    g = torch.Generator().manual_seed(8)
    M, N, K = 4, 5, 6
    x, w, b, c = (torch.randn(s, generator=g) for s in ((M, K), (N, K), (N,), (M, N)))
    for name in ("none", "gelu", "silu"):
        _, z = fl.fb_affine(x.cuda(), w.cuda(), b.cuda(), activation=name, want_preact=True)
        got = [d(t) for t in fl.fb_affine_grad(c.cuda(), x.cuda(), w.cuda(), activation=name, preact=z)]

        def f(x, w, b):
            return float((act(x @ w.t() + b, name) * c.double()).sum())

        args = [t.double().clone() for t in (x, w, b)]
        step = 1e-5
        for t, want in zip(args, got):
            flat = t.view(-1)
            for i in range(flat.numel()):
                keep = flat[i].item()
                flat[i] = keep + step
                up = f(*args)
                flat[i] = keep - step
                down = f(*args)
                flat[i] = keep
                assert abs((up - down) / (2 * step) - want.reshape(-1)[i].item()) <= 2e-5


def test_infinities_and_nan_stay_where_they_are(fl):
    """A row of x with NaN or inf spoils its row of y alone, a row of weight its column; so at every kernel's sizes."""
    import torch
    for M, N, K in [(3, 40, 24), (100, 90, 70), (600, 520, 264)]:
        for dtype in ("float32", "bfloat16"):
            x, w = rows(M, K, dtype, 0, 1), rows(N, K, dtype, 0, 2)
            x[1, K - 1] = math.nan
            w[N - 1, 0] = math.inf
            y = fl.fb_affine(x, w, activation="relu", out_dtype=torch.float32)
            bad = ~torch.isfinite(y)
            assert bad[1].all() and torch.isnan(y[1, :-1]).all()
            bad[1] = False
            assert not bad[:, :-1].any()
            neg = x[:, 0] < 0
            assert (y[:, -1][neg & (torch.arange(M, device="cuda") != 1)] == 0).all()


def test_no_rows_leading_shapes_and_another_stream(fl):
    import torch
    w = rows(20, 30, "float32", 0, 1)
    x = torch.empty((0, 30), device="cuda")
    assert fl.fb_affine(x, w).shape == (0, 20)
    dx, dw, db = fl.fb_affine_grad(torch.empty((0, 20), device="cuda"), x, w)
    assert dx.shape == (0, 30) and torch.equal(dw, torch.zeros_like(w)) and torch.equal(db, torch.zeros(20, device="cuda"))
    for n in (12, 3000):
        x = rows(n, 30, "float32", 0, 2)
        flat = fl.fb_affine(x, w)
        assert torch.equal(fl.fb_affine(x.view(n // 4, 4, 30), w).view(n, 20), flat)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            other = fl.fb_affine(x, w)
        s.synchronize()
        assert torch.equal(other, flat)


def test_outputs_beyond_32_bit_offsets(fl):
    """An output of more than 2^31 elements and of more than 4 GB."""
    import torch
    M, N, K = 1_100_000, 2048, 16
    x, w = torch.zeros((M, K), dtype=torch.bfloat16, device="cuda"), rows(N, K, "bfloat16", 0, 3)
    x[-300:] = rows(300, K, "bfloat16", 0, 4)
    y = fl.fb_affine(x, w)
    want = d(x[-300:]) @ d(w).t()
    assert ((d(y[-300:]) - want).abs() <= 2.0 ** -8 * want.abs() * 1.02 + 1e-4).all()
    assert not y[: M - 300: 997].any()
    dx, dw, db = fl.fb_affine_grad(y, x, w)
    want = d(y[-300:]).t() @ d(x[-300:])
    assert ((d(dw) - want).abs() <= 2.0 ** -7 * want.abs() + 1e-2).all()
    want = d(y[-300:]) @ d(w)
    assert ((d(dx[-300:]) - want).abs() <= 2.0 ** -7 * want.abs() + 1e-2).all()


@pytest.mark.parametrize("M,N,K", [(5, 300, 700), (600, 300, 520)])
def test_recorded_into_a_graph(fl, M, N, K):
    import torch
    x, w, dy = rows(M, K, "bfloat16", 0, 1), rows(N, K, "bfloat16", 0, 2), rows(M, N, "bfloat16", 0, 3)
    b = torch.ones(N, device="cuda")

    def step():
        y, z = fl.fb_affine(x, w, b, activation="gelu", want_preact=True)
        return (y, *fl.fb_affine_grad(dy, x, w, activation="gelu", preact=z))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for seed in (13, 14, 15):
        x.copy_(rows(M, K, "bfloat16", 0, seed))
        graph.replay()
        torch.cuda.synchronize()
        for a, c in zip(got, step()):
            assert torch.equal(a, c)


def test_refusals(fl):
    import torch
    x, w = torch.zeros((4, 8), device="cuda"), torch.zeros((6, 8), device="cuda")
    bad = [dict(x=x.cpu()), dict(x=x.double()), dict(weight=w[:, :7]), dict(weight=w.bfloat16()), dict(weight=w.view(-1)), dict(bias=torch.zeros(5, device="cuda")),
           dict(bias=torch.zeros(6, device="cuda", dtype=torch.float16)), dict(activation="tanh"), dict(residual=torch.zeros((4, 5), device="cuda")),
           dict(residual=torch.zeros((3, 6), device="cuda")), dict(out_dtype=torch.bfloat16), dict(x=x.t())]
    for change in bad:
        with pytest.raises(ValueError):
            fl.fb_affine(**{**dict(x=x, weight=w), **change})
    dy = torch.zeros((4, 6), device="cuda")
    for change in [dict(dy=dy[:3]), dict(dy=dy.half()), dict(activation="relu"), dict(activation="relu", preact=dy.half()), dict(weight=w[:5])]:
        with pytest.raises(ValueError):
            fl.fb_affine_grad(**{**dict(dy=dy, x=x, weight=w), **change})
    with pytest.raises(fl.FBError):
        fl.fb_affine(torch.zeros((4, 0), device="cuda"), torch.zeros((6, 0), device="cuda"))
