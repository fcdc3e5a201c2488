"""Gradients of half-precision affine layers whose dy is far smaller or larger than half precision reaches, against the
definition in 64 bits.

Tolerances.  u = 2^-24, h = 2^-11.  dz goes into the products times a power of two that brings the largest of dy into
[2^14, 2^15): its rounding is h of its size, and 2^-25 where that is below half precision's normal numbers, which taken back is at
most 2^-25 peak / 2^14 = 2^-39 peak.  Sums of K products have at most 300 + K / 16 roundings behind one another, each of at most
2 u of what is summed; the result is rounded once, h of its size or 2^-24 near 0.  That the bounds say something is held too:
they are small beside the result, in the 2-norm."""
from __future__ import annotations

import math

import pytest

pytestmark = pytest.mark.gpu

U, H, TINY = 2.0 ** -24, 2.0 ** -11, 2.0 ** -24


@pytest.fixture(scope="module")
def fl():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_2112_00709_amd as base
    from paper_2112_00709_amd import layers
    layers.lib()
    base.POISON_NEW_BUFFERS = True
    return layers


def d(t):
    return t.double().cpu()


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


def make(M, N, K, dy, dy_type, gap, seed):
    """x and weight such that the gradients lie well inside half precision, whatever the size of dy."""
    import torch
    g = torch.Generator().manual_seed(seed)

    def rows(n, width, t, scale, shift=0.0):
        a = torch.full((n, width + gap), math.nan)
        a[:, :width] = torch.randn((n, width), generator=g) * scale + shift
        return a.to(t).cuda()[:, :width]

    want = 30.0                                            # the size of the gradients that is aimed at
    x = rows(M, K, torch.float16, min(2000.0, max(1e-5, want / (dy * math.sqrt(M)))))
    w = rows(N, K, torch.float16, min(2000.0, max(1e-5, want / (dy * math.sqrt(N)))))
    return x, w, rows(M, N, dy_type, dy), rows(M, N, torch.float16, 1.0, 0.3)


def check(fl, x, w, dy, z, activation):
    import torch
    dx, dw, db = fl.fb_affine_grad(dy, x, w, activation=activation, preact=z if activation != "none" else None)
    M, N = dy.shape
    g = d(dy) * slope(d(z), activation)
    peak = d(dy).abs().max().item()
    eg = g.abs() * (H * 1.01 + 4 * U) + 16 * U * d(dy).abs() + 2.0 ** -39 * peak

    def held(got, want, tol):
        tol = tol * 1.01 + H * want.abs() * 1.01 + TINY
        bad = ~((d(got) - want).abs() <= tol)
        assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist(), d(got)[bad][:4], want[bad][:4])
        return (d(got) - want).norm() / want.norm()

    errors = [held(dx, g @ d(w), 2 * (300 + N / 16) * U * (g.abs() @ d(w).abs()) + eg @ d(w).abs()),
              held(dw, g.t() @ d(x), 2 * (300 + M / 16) * U * (g.abs().t() @ d(x).abs()) + eg.t() @ d(x).abs())]
    # the roundings of dz and of the result are each at most h of their size (terms that are alike round alike): 2 h in the 2-norm,
    # and what is smaller than half precision's normal numbers has its own
    for e, want in zip(errors, (g @ d(w), g.t() @ d(x))):
        assert e <= 2.1 * H + TINY * math.sqrt(want.numel()) / want.norm(), e
    tol = (300 + M / 16) * U * g.abs().sum(0) + (g.abs() * 4 * U + 16 * U * d(dy).abs()).sum(0)
    assert ((d(db) - g.sum(0)).abs() <= tol + 1e-37).all()
    assert torch.isfinite(dx).all() and torch.isfinite(dw).all()


# sizes of every way the products are laid out: few tiles in one launch, shares of k that are joined, tiles of 64 to 256
@pytest.mark.parametrize("M,N,K", [(1, 40, 24), (9, 51, 30), (65, 3, 70), (200, 84, 512), (3000, 300, 200), (1100, 520, 264), (8192, 96, 72)])
@pytest.mark.parametrize("activation", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("dy", [1e-8, 3e-6, 1.0, 1e6])
def test_single_precision_dy_of_any_size(fl, M, N, K, activation, dy):
    import torch
    check(fl, *make(M, N, K, dy, torch.float32, 0 if M % 2 else 5, M + N), activation)


@pytest.mark.parametrize("activation", ["gelu", "silu"])
@pytest.mark.parametrize("dy", [2e-7, 1e-5, 1.0, 15000.0])
def test_half_precision_dy_times_a_slope(fl, activation, dy):
    import torch
    for M, N, K in ((9, 51, 30), (3000, 300, 200)):
        x, w, g, z = make(M, N, K, dy, torch.float16, 0, M)
        g.clamp_(-65504, 65504)
        check(fl, x, w, g, z, activation)


def test_the_smallest_and_the_largest_half_precision_dy(fl):
    """Slopes below 1 on the smallest numbers there are, slopes above 1 on the largest."""
    import torch
    M, N, K = 4096, 64, 40
    x, w, _, z = make(M, N, K, 2.0 ** -24, torch.float16, 0, 1)
    dy = torch.full((M, N), 2.0 ** -24, device="cuda", dtype=torch.float16)
    x += 200.0
    w += 100.0
    z.fill_(-0.1)                                          # gelu's slope here: 0.42
    check(fl, x, w, dy, z, "gelu")
    dy.fill_(65504.0)
    z.fill_(1.4)                                           # 1.13
    check(fl, (x / 4e6).half(), (w / 2e5).half(), dy, z, "gelu")


def test_posterior_differences_divided_by_the_frames(fl):
    """What the objective hands a half-precision output layer: differences of posteriors, most of them tiny, over the frames."""
    import torch
    g = torch.Generator().manual_seed(2)
    M, N, K = 8192, 300, 128
    p, q = (torch.softmax(4 * torch.randn((M, N), generator=g), 1) for _ in range(2))
    dy = ((p - q) / 44152).cuda()
    x = (1 + torch.randn((M, K), generator=g)).half().cuda()
    w = (torch.randn((N, K), generator=g) * 300).half().cuda()
    check(fl, x, w, dy, torch.zeros((M, N), device="cuda").half(), "none")


def test_zeros_denormals_and_infinities_in_dy(fl):
    import torch
    for M, N, K in ((5, 40, 24), (700, 120, 88)):
        x, w, dy, z = make(M, N, K, 1e-6, torch.float32, 0, 3)
        for zero in (torch.zeros_like(dy), torch.full_like(dy, 1e-42)):
            dx, dw, db = fl.fb_affine_grad(zero, x, w)
            assert not dx.any() and not dw.any()
        dx, dw, db = fl.fb_affine_grad(dy, x, w)
        for bad in (math.inf, math.nan):                   # a row that is lost takes no other row with it
            dy2 = dy.clone()
            dy2[2, 3] = bad
            dx2 = fl.fb_affine_grad(dy2, x, w)[0]
            keep = torch.arange(M, device="cuda") != 2
            assert not torch.isfinite(dx2[2]).any()
            assert ((d(dx2) - d(dx))[keep.cpu()].abs() <= 4 * H * d(dx)[keep.cpu()].abs() + 2.0 ** -38 * d(dy).abs().max() * d(w).abs().sum(0) + TINY).all()


def test_parts_of_the_gradient_and_no_rows(fl):
    import torch
    x, w, dy, z = make(3000, 300, 200, 1e-7, torch.float32, 0, 4)
    full = fl.fb_affine_grad(dy, x, w, activation="silu", preact=z)
    for want in [(True, False, False), (False, True, False), (False, False, True), (True, False, True)]:
        got = fl.fb_affine_grad(dy, x, w, activation="silu", preact=z, want_dx=want[0], want_dweight=want[1], want_dbias=want[2])
        for a, b, asked in zip(got, full, want):
            assert (a is None) == (not asked)
            assert not asked or torch.equal(a, b)
    dx, dw, db = fl.fb_affine_grad(dy[:0], x[:0], w, activation="silu", preact=z[:0])
    assert dx.shape == (0, 200) and not dw.any() and not db.any()


def test_recorded_into_a_graph_with_dy_of_other_sizes_later(fl):
    import torch
    x, w, dy, z = make(600, 300, 520, 1e-3, torch.float32, 0, 5)

    def step():
        return fl.fb_affine_grad(dy, x, w, activation="gelu", preact=z)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    first = dy.clone()
    for scale in (1.0, 1e-4, 100.0, 1e-3):
        dy.copy_(first * scale)
        graph.replay()
        torch.cuda.synchronize()
        for a, c in zip(got, step()):
            assert torch.equal(a, c)


def test_small_factors_of_the_forward_product(fl):
    """Half-precision inputs below its normal numbers are numbers all the same: their products have no error of their own."""
    import torch
    g = torch.Generator().manual_seed(6)
    for M, N, K in ((3, 40, 64), (300, 136, 200)):
        x = (torch.randn((M, K), generator=g) * 1e-6).half().cuda()
        w = (torch.randn((N, K), generator=g) * 500).half().cuda()
        y = fl.fb_affine(x, w, out_dtype=torch.float32)
        want, size = d(x) @ d(w).t(), d(x).abs() @ d(w).abs().t()
        assert ((d(y) - want).abs() <= 2 * (300 + K / 16) * U * size).all() and size.min() > 1e-4
