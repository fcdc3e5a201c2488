"""Layer norm and its gradient on the GPU against the definition in 64 bits.

Tolerances.  u = 2^-24 is single precision's unit roundoff, h the type's own (2^-24, 2^-8 for bfloat16, 2^-11 for half with
2^-25 absolute where it is denormal).  A sum of H terms over lanes and a fixed tree has at most H / 64 + 16 roundings one after the other (less in every kernel
here), so the mean is off by at most n u mean|x| and so on; with n = 300 for the widths below a bound of 300 u relative to
the sums of absolute values holds, to which the type's rounding of the result is added."""
from __future__ import annotations

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
H_OF = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
N_ROUND = 300


@pytest.fixture(scope="module")
def fl():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_2112_00709_amd as base
    from paper_2112_00709_amd import layers
    layers.lib()
    base.POISON_NEW_BUFFERS = True   # outputs and workspaces start out as NaN
    return layers


def make(R, H, dtype, gap, seed, offset=0.0, scale=1.5):
    import torch
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn((R, H + gap), generator=g) * scale + torch.randn((R, 1), generator=g) + offset).to(getattr(torch, dtype))
    return x.cuda()[:, :H]


def definition(x, w, b, eps):
    xd = x.double().cpu()
    mean = xd.mean(1)
    d = xd - mean[:, None]
    var = (d * d).mean(1)
    rstd = 1 / (var + eps).sqrt()
    y = d * rstd[:, None]
    if w is not None:
        y = y * w.double().cpu()
    if b is not None:
        y = y + b.double().cpu()
    return y, mean, rstd


SHAPES = [(1, 1), (1, 2), (3, 7), (5, 64), (4, 97), (9, 511), (2, 512), (7, 513), (130, 1000), (6, 1024), (5, 1025), (3, 2048), (4, 2051), (3, 4096),
          (2, 4099), (3, 8192), (2, 8200), (2, 16384), (3, 16385), (1, 40001)]


@pytest.mark.parametrize("R,H", SHAPES)
@pytest.mark.parametrize("dtype,wdtype,gap", [("float32", "float32", 0), ("bfloat16", "float32", 3), ("float16", "float16", 1), ("bfloat16", "bfloat16", 0)])
def test_forward_and_gradient(fl, R, H, dtype, wdtype, gap):
    import torch
    eps = 1e-5
    x = make(R, H, dtype, gap, 3 * R + H)
    g = torch.Generator().manual_seed(H)
    w = (1 + 0.3 * torch.randn(H, generator=g)).to(getattr(torch, wdtype)).cuda()
    b = (0.2 * torch.randn(H, generator=g)).to(getattr(torch, wdtype)).cuda()
    dy = (0.7 * torch.randn((R, H + gap), generator=g)).to(x.dtype).cuda()[:, :H]
    y, mean, rstd = fl.fb_layer_norm(x, w, b, eps, want_stats=True)
    ry, rmean, rrstd = definition(x, w, b, eps)
    xd = x.double().cpu()
    absmean = xd.abs().mean(1)
    h = H_OF[dtype]
    tiny = 2.0 ** -24 if dtype == "float16" else 0.0
    # the mean's error e shifts every distance from it by e and, with the variance's, scales them
    e_mean = N_ROUND * U * absmean + 1e-30
    assert ((mean.double().cpu() - rmean).abs() <= e_mean).all()
    e_rstd = rrstd * (N_ROUND * U + e_mean ** 2 * rrstd ** 2 + 2 * U)
    assert ((rstd.double().cpu() - rrstd).abs() <= e_rstd).all()
    wa = w.double().cpu().abs()
    e_y = wa * (e_mean[:, None] * rrstd[:, None] * 1.1 + (N_ROUND * U + e_mean[:, None] ** 2 * rrstd[:, None] ** 2) * ((xd - rmean[:, None]).abs() * rrstd[:, None])) + 4 * U * b.double().cpu().abs()
    assert ((y.double().cpu() - ry).abs() <= 1.1 * e_y + h * ry.abs() + tiny).all()
    assert y.dtype == x.dtype and y.shape == x.shape

    # the gradient takes the statistics as they were handed over
    dx, dw, db = fl.fb_layer_norm_grad(dy, x, mean, rstd, w)
    m, s = mean.double().cpu()[:, None], rstd.double().cpu()[:, None]
    xh, dyd, wd = (xd - m) * s, dy.double().cpu(), w.double().cpu()
    gg = dyd * wd
    want = s * (gg - gg.mean(1, keepdim=True) - xh * (gg * xh).mean(1, keepdim=True))
    # distances of x from a mean of about its size lose up to u |x| s each: e_xh
    e_xh = 3 * U * (xd.abs() + m.abs()) * s + 3 * U * xh.abs()
    c1 = (gg * xh).mean(1, keepdim=True).abs()
    e_dx = s * (N_ROUND * U * (gg.abs() + gg.abs().mean(1, keepdim=True) + xh.abs() * (gg * xh).abs().mean(1, keepdim=True))
                + e_xh * c1 + xh.abs() * (gg.abs() * e_xh).mean(1, keepdim=True))
    assert ((dx.double().cpu() - want).abs() <= 1.1 * e_dx + h * want.abs() + tiny).all()
    e_dw = N_ROUND * U * (dyd * xh).abs().sum(0) + (dyd.abs() * e_xh).sum(0)
    assert ((dw.double().cpu() - (dyd * xh).sum(0)).abs() <= 1.1 * e_dw + 1e-30).all()
    assert ((db.double().cpu() - dyd.sum(0)).abs() <= N_ROUND * U * dyd.abs().sum(0) + 1e-30).all()
    assert dw.dtype == torch.float32 and db.dtype == torch.float32


@pytest.mark.parametrize("H", [5, 512, 777, 3001, 20000])
def test_many_rows_sums_do_not_depend_on_what_else_is_wanted(fl, H):
    """Several rows a workgroup; outputs left out leave the others as they are, and a second call gives the same bits."""
    import torch
    R = 5003 if H < 1000 else 1201
    x, dy = make(R, H, "bfloat16", 0, 1), make(R, H, "bfloat16", 0, 2)
    w = torch.linspace(0.5, 1.5, H, device="cuda")
    _, mean, rstd = fl.fb_layer_norm(x, w, None, want_stats=True)
    dx, dw, db = fl.fb_layer_norm_grad(dy, x, mean, rstd, w)
    xh = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    ref, scale = (dy.double() * xh).sum(0), (dy.double() * xh).abs().sum(0)
    # at most R / 512 + 16 + 32 roundings behind one another, and those of a distance from the mean
    assert ((dw.double() - ref).abs() <= 60 * U * scale + 6 * U * ((x.double().abs() + mean.double().abs()[:, None]) * rstd.double()[:, None] * dy.double().abs()).sum(0)).all()
    assert ((db.double() - dy.double().sum(0)).abs() <= 60 * U * dy.double().abs().sum(0)).all()
    for want in [(True, False, False), (False, True, False), (False, False, True), (False, True, True)]:
        got = fl.fb_layer_norm_grad(dy, x, mean, rstd, w, *want)
        for g, full, asked in zip(got, (dx, dw, db), want):
            assert (g is None) == (not asked)
            if asked:
                assert torch.equal(g, full)


def test_without_weight_and_rows_of_equal_elements(fl):
    import torch
    x = torch.full((3, 100), 7.25, device="cuda")
    y, mean, rstd = fl.fb_layer_norm(x, eps=1e-5, want_stats=True)
    # sums of 100 equal numbers: 7.25 * 100 is exact in every order, the division by 100 rounds once or twice
    assert (mean - 7.25).abs().max() <= 7.25 * 2 * U and (y.abs() <= 7.25 * 4 * U * 317).all()
    assert torch.allclose(rstd, torch.full_like(rstd, 1e-5 ** -0.5), rtol=1e-4)
    b = torch.arange(100, device="cuda", dtype=torch.float32)
    assert (fl.fb_layer_norm(x, None, b) - b).abs().max() <= 7.25 * 4 * U * 317 + 100 * U
    dx, dw, db = fl.fb_layer_norm_grad(torch.ones_like(x), x, mean, rstd)
    assert dx.abs().max() <= 1e-3 and torch.equal(db, torch.full_like(db, 3.0))


def test_gradient_against_differences(fl):
    """dx, dweight and dbias against central differences of a 64-bit evaluation of the definition."""
    import torch
    g = torch.Generator().manual_seed(5)
    R, H, eps = 3, 17, 1e-5
    x, c = torch.randn((R, H), generator=g), torch.randn((R, H), generator=g)
    w, b = 1 + 0.3 * torch.randn(H, generator=g), torch.randn(H, generator=g)
    xg, wg = x.cuda(), w.cuda()
    _, mean, rstd = fl.fb_layer_norm(xg, wg, b.cuda(), eps, want_stats=True)
    dx, dw, db = (t.double().cpu() for t in fl.fb_layer_norm_grad(c.cuda(), xg, mean, rstd, wg))

    def f(x, w, b):
        return float((definition(x, w, b, eps)[0] * c.double()).sum())

    step = 1e-5                                   # third derivatives of order 10: the differences are good to 1e-8
    x, w, b = x.double(), w.double(), b.double()
    for t, got in ((x, dx), (w, dw), (b, db)):
        flat, got = t.view(-1), got.reshape(-1)
        for i in range(0, flat.numel(), 3):
            keep = flat[i].item()
            flat[i] = keep + step
            up = f(x, w, b)
            flat[i] = keep - step
            down = f(x, w, b)
            flat[i] = keep
            assert abs((up - down) / (2 * step) - got[i].item()) <= 2e-5


def test_no_rows_leading_shapes_and_another_stream(fl):
    import torch
    x = torch.empty((0, 33), device="cuda")
    y, mean, rstd = fl.fb_layer_norm(x, want_stats=True)
    assert y.shape == (0, 33) and mean.shape == (0,)
    dx, dw, db = fl.fb_layer_norm_grad(x, x, mean, rstd)
    assert torch.equal(dw, torch.zeros(33, device="cuda")) and torch.equal(db, torch.zeros(33, device="cuda"))
    x = make(12, 50, "float32", 0, 9)
    flat = fl.fb_layer_norm(x)
    assert torch.equal(fl.fb_layer_norm(x.view(3, 4, 50)).view(12, 50), flat)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = fl.fb_layer_norm(x)
    s.synchronize()
    assert torch.equal(other, flat)


def test_rows_beyond_32_bit_offsets(fl):
    """The last rows of 2^31 and more elements (4.3 GB)."""
    import torch
    H, R = 1024, (1 << 21) + 5
    x = torch.zeros((R, H), dtype=torch.bfloat16, device="cuda")
    x[-3:] = make(3, H, "bfloat16", 0, 4)
    y, mean, rstd = fl.fb_layer_norm(x, want_stats=True)
    ry, rmean, _ = definition(x[-3:], None, None, 1e-5)
    assert (mean[-3:].double().cpu() - rmean).abs().max() <= 1e-5
    assert (y[-3:].double().cpu() - ry).abs().max() <= 2.0 ** -7 * ry.abs().max()
    dx, _, db = fl.fb_layer_norm_grad(x, x, mean, rstd)
    assert ((db.double() - x.double()[-3:].sum(0)).abs() <= 1e-5 * x.double()[-3:].abs().sum(0) + 1e-12).all()
    assert dx[-3:].float().abs().max() < 1.0 and torch.isfinite(dx[-3:]).all()


def test_recorded_into_a_graph(fl):
    import torch
    x, dy = make(70, 300, "bfloat16", 0, 11), make(70, 300, "bfloat16", 0, 12)
    w = torch.linspace(0.5, 1.5, 300, device="cuda")

    def step():
        y, mean, rstd = fl.fb_layer_norm(x, w, want_stats=True)
        return (y, *fl.fb_layer_norm_grad(dy, x, mean, rstd, w))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for seed in (13, 14, 15):
        x.copy_(make(70, 300, "bfloat16", 0, seed))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, step()):
            assert torch.equal(a, b)


def test_refusals(fl):
    import torch
    x = torch.zeros((4, 8), device="cuda")
    with pytest.raises(ValueError):
        fl.fb_layer_norm(torch.zeros((4, 8)))                                   # not on the GPU
    with pytest.raises(ValueError):
        fl.fb_layer_norm(x.double())
    with pytest.raises(ValueError):
        fl.fb_layer_norm(x.t())                                                 # elements of a row apart
    with pytest.raises(ValueError):
        fl.fb_layer_norm(x, torch.ones(7, device="cuda"))
    with pytest.raises(ValueError):
        fl.fb_layer_norm(x, torch.ones(8, device="cuda"), torch.ones(8, device="cuda", dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        fl.fb_layer_norm(x, torch.ones(8, device="cuda", dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        fl.fb_layer_norm(torch.zeros((4, 4, 8), device="cuda")[:, :3])          # rows at two distances
    for eps in (-1.0, float("nan"), float("inf")):
        with pytest.raises(fl.FBError) as err:
            fl.fb_layer_norm(x, eps=eps)
        assert err.value.code == -1
    _, mean, rstd = fl.fb_layer_norm(x, want_stats=True)
    with pytest.raises(ValueError):
        fl.fb_layer_norm_grad(x[:3], x, mean, rstd)
    with pytest.raises(ValueError):
        fl.fb_layer_norm_grad(x, x, mean[:3], rstd)
    with pytest.raises(fl.FBError):
        fl.fb_layer_norm(torch.zeros((4, 0), device="cuda"))
