"""Gradients of few rows in 16 bits: what is rounded before the products is kept in two numbers, so that the gradients are off by little more
than their own rounding, whatever a single row's largest slope is."""
from __future__ import annotations

import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def fl():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_2112_00709_amd as base
    from paper_2112_00709_amd import layers
    layers.lib()
    base.POISON_NEW_BUFFERS = True
    return layers


def numbers(shape, seed, dtype="float32", scale=1.0):
    import torch
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).cuda().to(getattr(torch, dtype))


def check(got, want, off, dtype):
    """One rounding to the type (half a step: eps / 2) and `off` before it; half precision's steps do not get smaller than 2^-25 each side."""
    import torch
    t = getattr(torch, dtype)
    half = torch.finfo(t).eps / 2 if got.dtype == t else 2 * U
    tol = (off + half * (want.abs() + off)) * 1.001 + (2.0 ** -25 if got.dtype == torch.float16 else 0.0)
    assert got.shape == want.shape and torch.isfinite(got).all()
    assert ((got.double() - want).abs() <= tol).all()


def products(dz, off, x, w, dtype):
    """dx, dw in 64 bits and how far off the sums may be: dz by `off` and, kept in two, by half a step of half a step; each of n sums' terms
    by one rounding of the running sum."""
    import torch
    half = torch.finfo(getattr(torch, dtype)).eps / 2
    off = off + dz.abs() * half * half * 1.01
    dx, dw = dz @ w, dz.t().contiguous() @ x
    ex = (off + (dz.abs() + off) * (2 * dz.shape[1] + 16) * U) @ w.abs()
    ew = (off + (dz.abs() + off) * (2 * dz.shape[0] + 16) * U).t().contiguous() @ x.abs()
    return dx, ex, dw, ew


ROWS = [1, 2, 3, 17, 31, 32, 33, 63, 64, 65, 95, 127, 128]


def sizes(twice, others):
    """Rows up to 64, and beyond in small products alone (`twice`: N stands for 2 N rows of the weight)."""
    return [(M, N, K) for N, K in others for M in ROWS if M <= 64 or M * twice * N * K <= 2 ** 24]


@pytest.mark.parametrize("M,N,K", sizes(2, [(5, 3), (64, 128), (77, 35), (515, 264)]))
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_gated_layer(fl, M, N, K, dtype):
    import torch
    x, w, z, dy = numbers((M, K), 1, dtype), numbers((2 * N, K), 2, dtype, K ** -0.5), numbers((M, 2 * N), 3, dtype), numbers((M, N), 4, dtype, 0.1)
    dx, dw, db = fl.fb_gated_affine_grad(dy, x, w, z, activation="silu")
    d, (g, u) = dy.double(), z.double().chunk(2, 1)
    s = torch.sigmoid(g)
    dz = torch.cat([d * u * s * (1 + g * (1 - s)), d * g * s], 1)
    off = torch.cat([(d * u).abs() * (4 + g.abs() * 4), (d * g).abs() * 4], 1) * 4 * U        # (exponential, reciprocal, products: four steps)
    wx, ex, ww, ew = products(dz, off, x.double(), w.double(), dtype)
    check(dx, wx, ex, dtype)
    check(dw, ww, ew, dtype)
    check(db, dz.sum(0), (off + dz.abs() * (M + 4) * U).sum(0), dtype)
    for want in [(True, False, False), (False, True, False), (True, False, True), (False, True, True)]:
        for p, q in zip(fl.fb_gated_affine_grad(dy, x, w, z, "silu", *want), (dx, dw, db)):
            assert p is None or torch.equal(p, q)


@pytest.mark.parametrize("M,V,K", sizes(1, [(3, 5), (40, 128), (1083, 29), (2050, 264)]) + [(3, 2_200_000, 16), (40, 2_100_001, 9)])
@pytest.mark.parametrize("dtype,entropy", [("bfloat16", True), ("float16", True), ("bfloat16", False)])
def test_log_probabilities(fl, M, V, K, dtype, entropy):
    import torch
    x, w, b = numbers((M, K), 1, dtype), numbers((V, K), 2, dtype, 2 * K ** -0.5), numbers(V, 3, scale=0.5)
    tokens = torch.randint(0, V, (M,), generator=torch.Generator().manual_seed(M), dtype=torch.int32).cuda()
    if M > 2:
        tokens[[1, M - 1]] = -1                             # rows that do not count may hold anything
        x[1] = float("nan")
    live = tokens >= 0
    lp, ent, logz = fl.fb_affine_logprobs(x, w, tokens, b)
    g, h = numbers(M, 5) * 0.1 - 1, numbers(M, 6) * 0.1 if entropy else None
    dx, dw, db = fl.fb_affine_logprobs_grad(x, w, tokens, logz, ent, g, h, b)
    xd, wd = x.double().masked_fill(~live[:, None], 0), w.double()
    z = xd @ wd.t().contiguous() + b.double()
    ez = (xd.abs() @ wd.t().abs().contiguous() + b.abs().double()) * (K + 4) * U + 8 * U * (z.abs() + logz.double().abs()[:, None] + 1)
    logp = z - logz.double()[:, None]
    p, hd = logp.exp(), h.double()[:, None] if entropy else torch.zeros((M, 1), dtype=torch.float64, device="cuda")
    e, gd = ent.double()[:, None], g.double()[:, None]
    dz = -p * (gd + hd * (logp + e))
    off = (p * (gd.abs() + hd.abs() * (logp.abs() + e.abs() + 1))) * (1.01 * ez + 16 * U)
    dz.scatter_add_(1, tokens.clamp_min(0).long()[:, None], gd)
    off = (off + 2 * U * (dz.abs() + gd.abs() * 0)).masked_fill(~live[:, None], 0)
    dz = dz.masked_fill(~live[:, None], 0)
    wx, ex, ww, ew = products(dz, off, xd, wd, dtype)
    check(dx, wx, ex, dtype)
    check(dw, ww, ew, dtype)
    check(db, dz.sum(0), (off + dz.abs() * (M + 4) * U).sum(0), dtype)
    for want in [(True, False, False), (False, True, False), (True, False, True), (False, True, True)]:
        for q, r in zip(fl.fb_affine_logprobs_grad(x, w, tokens, logz, ent, g, h, b, *want), (dx, dw, db)):
            assert q is None or torch.equal(q, r)


@pytest.mark.parametrize("M,V,K", [(62, 300, 3834), (192, 186, 3769), (700, 128, 1216)])
def test_long_sums_in_single_precision(fl, M, V, K):
    """Logits' sums over a long k are added up in shares of 256: log Z and the gradient are off by what sums of 256 + K / 256 terms are."""
    import torch
    x, w = numbers((M, K), 1), numbers((V, K), 2, scale=2 * K ** -0.5)
    tokens = torch.randint(0, V, (M,), generator=torch.Generator().manual_seed(M), dtype=torch.int32).cuda()
    lp, ent, logz = fl.fb_affine_logprobs(x, w, tokens)
    z = x.double() @ w.double().t().contiguous()
    terms = (256 + K / 256 + 8) * U * (x.abs().double() @ w.abs().double().t().contiguous()) if M > 64 else K * U * (x.abs().double() @ w.abs().double().t().contiguous())
    ez = terms.max(1).values + 8 * U * (z.abs().max(1).values + 8)
    assert ((logz.double() - z.logsumexp(1)).abs() <= ez).all()
    g = numbers(M, 5) * 0.1 - 1
    _, _, db = fl.fb_affine_logprobs_grad(x, w, tokens, logz, None, g, None, None)
    dz = -torch.softmax(z, 1) * g.double()[:, None]
    e = (dz.abs() * (2 * ez[:, None] + 16 * U)).sum(0)
    dz.scatter_add_(1, tokens.long()[:, None], g.double()[:, None])
    assert ((db.double() - dz.sum(0)).abs() <= e + dz.abs().sum(0) * (M + 4) * U + g.abs().sum().double() * 4 * U).all()
