"""The way from one block into the next (norm, gate, scale, residual, norm) and its gradient on the GPU against the definition in
64 bits.

Tolerances.  u = 2^-24, h the type's roundoff.  A mean over a row is formed with at most 40 roundings one after the other (16
elements a lane, 6 steps over a wave, 8 waves), a sum over R rows with at most 60 + R / 256 (rows a lane sees, workgroups' rows in
64ths).  The bounds below carry the error of each step into the next by its derivative, every product and sum with its own u;
the result is rounded once: h."""
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


def rows(n, width, dtype, gap, seed, scale=1.0, shift=0.0):
    """Rows of a wider tensor; what lies between them is NaN."""
    import torch
    g = torch.Generator().manual_seed(seed)
    x = torch.full((n, width + gap), math.nan)
    x[:, :width] = torch.randn((n, width), generator=g) * scale + shift * torch.randn((n, 1), generator=g)
    return x.to(getattr(torch, dtype)).cuda()[:, :width]


def vector(n, dtype, seed, scale, shift):
    import torch
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(n, generator=g) * scale + shift).to(getattr(torch, dtype)).cuda()


def d(t):
    return t.double().cpu()


def make(R, H, dtype, gap, inner, outer, gate, residual, wdtype, seed=0):
    c = dict(scale=0.7, inner=inner, outer=outer)
    h = rows(R, H, dtype, gap, seed + 1, 0.8, 0.3)
    r = rows(R, H, dtype, gap, seed + 2, 1.5) if residual else None
    g = vector(H, wdtype, seed + 3, 0.2, 0.5) if gate == "vector" else rows(R, H, dtype, gap, seed + 3, 0.3) if gate == "rows" else None
    if inner != "none" and seed % 3 != 2:
        c.update(inner_weight=vector(H, wdtype, seed + 4, 0.2, 1), inner_bias=vector(H, wdtype, seed + 5, 0.1, 0) if seed % 2 else None)
    if outer != "none" and seed % 3 != 1:
        c.update(weight=vector(H, wdtype, seed + 6, 0.2, 1), bias=vector(H, wdtype, seed + 7, 0.1, 0) if seed % 2 == 0 else None)
    return h, r, g, c


def one(v, none):
    import torch
    return torch.full((1,), float(none), dtype=torch.float64) if v is None else d(v)


def norm(x, ex, kind, w, b, eps):
    """-> (y, its error, xh, mean, rstd, error of mean, relative error of rstd) of rows known up to ex."""
    import torch
    H = x.shape[1]
    mean, em = torch.zeros(len(x), 1).double(), torch.zeros(len(x), 1).double()
    if kind == "none":
        return x, ex, x, mean, mean + 1, em, em
    if kind == "layer":
        mean, em = x.mean(1, keepdim=True), ex.mean(1, keepdim=True) + 42 * U * x.abs().mean(1, keepdim=True)
    t = x - mean
    e = ex + em + U * (x.abs() + mean.abs())
    var = t.square().mean(1, keepdim=True)
    evar = 2 * (t.abs() * e).mean(1, keepdim=True) + e.square().mean(1, keepdim=True) + 50 * U * var
    rstd = (var + eps).rsqrt()
    er = 0.5 * evar / (var + eps) + 5 * U
    xh = t * rstd
    exh = (e * rstd + xh.abs() * er) * 1.01 + 2 * U * xh.abs()
    return xh * w + b, w.abs() * exh + 4 * U * ((xh * w).abs() + b.abs()), xh, mean, rstd, em, er


def close(got, want, err, dtype, what):
    import torch
    tol = err + H_OF[dtype] * (want.abs() + err) * 1.01 + TINY[dtype]
    assert got.dtype == getattr(torch, dtype), what
    bad = ~((d(got) - want).abs() <= tol)
    assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[:4].tolist(), d(got)[bad][:4], want[bad][:4], tol[bad][:4])


def check_forward(fl, R, H, dtype, gap, inner, outer, gate, residual, wdtype, seed=0, eps=1e-5):
    import torch
    h, r, g, c = make(R, H, dtype, gap, inner, outer, gate, residual, wdtype, seed)
    s, y, stats = fl.fb_residual_norm(h, r, g, eps=eps, want_stats=True, **c)
    s2, y2 = fl.fb_residual_norm(h, r, g, eps=eps, **c)
    assert torch.equal(s, s2) and (y is None) == (outer == "none") and (y is None or torch.equal(y, y2))
    f = one(g, 1) * c["scale"]
    x = d(h)
    u, eu, _, m1, r1, em1, er1 = norm(x, torch.zeros_like(x), inner, one(c.get("inner_weight"), 1), one(c.get("inner_bias"), 0), eps)
    res = d(r) if residual else torch.zeros_like(x)
    v = res + f * u
    ev = f.abs() * eu + 8 * U * (f.abs() * (u.abs() + one(c.get("inner_bias"), 0).abs() * 2) + res.abs())
    close(s, v, ev, dtype, "s")
    want, e, _, m2, r2, em2, er2 = norm(v, ev, outer, one(c.get("weight"), 1), one(c.get("bias"), 0), eps)
    if outer != "none":
        close(y, want, e, dtype, "y")
    for k, (a, b) in enumerate([(m1, em1), (r1, r1 * er1), (m2, em2), (r2, r2 * er2)]):
        close(stats[k], a[:, 0], b[:, 0] + 2 * U * a[:, 0].abs(), "float32", f"stats {k}")


SIZES = [(1, 1), (1, 512), (2, 3), (5, 64), (7, 777), (3, 513), (130, 512), (33, 1000), (9, 1024), (5, 1025), (6, 2000), (4, 2048), (3, 2049), (7, 4096),
         (2, 4097), (5, 8191), (3, 8192), (2100, 40), (1500, 520)]
KINDS = [("rms", "rms", "vector", True), ("layer", "layer", "rows", True), ("none", "layer", "none", True), ("rms", "none", "rows", False),
         ("none", "rms", "vector", False), ("layer", "rms", "none", True), ("none", "none", "rows", True)]


@pytest.mark.parametrize("R,H", SIZES)
@pytest.mark.parametrize("dtype,gap,wdtype", [("float32", 0, "float32"), ("bfloat16", 0, "float32"), ("float16", 3, "float16"), ("bfloat16", 5, "bfloat16")])
def test_forward(fl, R, H, dtype, gap, wdtype):
    k = R + H
    for v in range(3):
        check_forward(fl, R, H, dtype, gap, *KINDS[(k + 2 * v) % 7], wdtype, seed=k + v)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("inner", ["none", "layer", "rms"])
@pytest.mark.parametrize("outer", ["none", "layer", "rms"])
def test_every_form(fl, dtype, inner, outer):
    for gate in ("none", "vector", "rows"):
        for residual in (False, True):
            check_forward(fl, 6, 200, dtype, 0, inner, outer, gate, residual, "float32", seed=len(inner) + len(outer))
            check_grad(fl, 6, 200, dtype, 0, inner, outer, gate, "float32", seed=len(inner) + len(outer))


def check_grad(fl, R, H, dtype, gap, inner, outer, gate, wdtype, seed=0, with_ds=True):
    import torch
    h, r, g, c = make(R, H, dtype, gap, inner, outer, gate, True, wdtype, seed)
    s, _, stats = fl.fb_residual_norm(h, r, g, want_stats=True, **c)
    c.pop("bias", None)
    ds = rows(R, H, dtype, gap, seed + 8, 0.2) if with_ds or outer == "none" else None
    dy = rows(R, H, dtype, gap, seed + 9, 0.2) if outer != "none" else None
    got = fl.fb_residual_norm_grad(ds, dy, h, s, stats, g, **c)
    m1, r1, m2, r2 = [t[:, None] for t in d(stats)]
    zero = torch.zeros((R, H)).double()
    total = d(ds) if ds is not None else zero
    size, e = total.abs(), zero
    n = 60 + R / 256
    want = [None] * 7
    if outer != "none":
        w2 = one(c.get("weight"), 1)
        xh, dyd = (d(s) - m2) * r2, d(dy)
        exh = 3 * U * (d(s).abs() + m2.abs()) * r2
        q = dyd * w2
        t0, t1 = q.mean(1, keepdim=True) if outer == "layer" else 0.0, (q * xh).mean(1, keepdim=True)
        total = total + r2 * (q - t0 - xh * t1)
        size = size + r2 * (q.abs() + q.abs().mean(1, keepdim=True) + xh.abs() * (q * xh).abs().mean(1, keepdim=True))
        e = r2 * (xh.abs() * (q.abs() * exh).mean(1, keepdim=True) + exh * t1.abs())
        want[5] = (dyd * xh).sum(0), (dyd.abs() * exh).sum(0) + n * U * (dyd * xh).abs().sum(0)
        want[6] = dyd.sum(0), n * U * dyd.abs().sum(0)
    e = e + 60 * U * size
    want[1] = total, e
    w1, b1 = one(c.get("inner_weight"), 1), one(c.get("inner_bias"), 0)
    xh = (d(h) - m1) * r1
    exh = 3 * U * (d(h).abs() + m1.abs()) * r1
    du, edu = total * c["scale"], e * c["scale"] + 2 * U * total.abs()
    if g is not None:
        u = xh * w1 + b1
        dg = du * u
        edg = edu * u.abs() + du.abs() * (w1.abs() * exh + 3 * U * ((xh * w1).abs() + b1.abs())) + 3 * U * dg.abs()
        want[2] = (dg.sum(0), edg.sum(0) + n * U * dg.abs().sum(0)) if gate == "vector" else (dg, edg)
        du, edu = du * d(g), edu * d(g).abs() + 2 * U * (du * d(g)).abs()
    want[0] = du, edu
    if inner != "none":
        want[3] = (du * xh).sum(0), (edu * xh.abs() + du.abs() * exh).sum(0) + n * U * (du * xh).abs().sum(0)
        want[4] = du.sum(0), edu.sum(0) + n * U * du.abs().sum(0)
        q, eq = du * w1, edu * w1.abs() + U * (du * w1).abs()
        t0, t1 = q.mean(1, keepdim=True) if inner == "layer" else 0.0, (q * xh).mean(1, keepdim=True)
        size = r1 * (q.abs() + q.abs().mean(1, keepdim=True) + xh.abs() * (q * xh).abs().mean(1, keepdim=True))
        e = r1 * (eq + eq.mean(1, keepdim=True) + xh.abs() * (eq * xh.abs()).mean(1, keepdim=True)
                  + xh.abs() * (q.abs() * exh).mean(1, keepdim=True) + exh * t1.abs())
        want[0] = r1 * (q - t0 - xh * t1), e + 60 * U * size
    for k, what in enumerate(("dh", "dresidual", "dgate", "dinner_weight", "dinner_bias", "dweight", "dbias")):
        assert (got[k] is None) == (want[k] is None), what
        if want[k] is not None:
            close(got[k], want[k][0], want[k][1], dtype if k < 2 or (k == 2 and gate == "rows") else "float32", what)
    return got


@pytest.mark.parametrize("R,H", SIZES)
@pytest.mark.parametrize("dtype,gap,wdtype", [("float32", 0, "float32"), ("bfloat16", 0, "float32"), ("float16", 3, "float16"), ("bfloat16", 5, "bfloat16")])
def test_gradient(fl, R, H, dtype, gap, wdtype):
    k = R + H
    for v in range(3):
        inner, outer, gate, _ = KINDS[(k + 2 * v) % 7]
        check_grad(fl, R, H, dtype, gap, inner, outer, gate, wdtype, seed=k + v, with_ds=v != 1)


def test_gradient_against_differences(fl):
    """(f(x + t e) - f(x - t e)) / 2t of the definition in 64 bits, along random directions of every input."""
    import torch
    R, H = 5, 70
    h, r, g, c = make(R, H, "float32", 0, "layer", "rms", "rows", True, "float32", seed=3)
    c["weight"] = vector(H, "float32", 50, 0.2, 1)
    c["inner_weight"], c["inner_bias"] = vector(H, "float32", 51, 0.2, 1), vector(H, "float32", 52, 0.2, 0)
    c["bias"] = None
    s, _, stats = fl.fb_residual_norm(h, r, g, want_stats=True, **c)
    c.pop("bias")
    ds, dy = rows(R, H, "float32", 0, 11), rows(R, H, "float32", 0, 12)
    got = fl.fb_residual_norm_grad(ds, dy, h, s, stats, g, **c)
    base = [d(t) for t in (h, r, g, c["inner_weight"], c["inner_bias"], c["weight"])]

    def value(h, r, g, w1, b1, w2):
        t = h - h.mean(1, keepdim=True)
        u = t / (t.square().mean(1, keepdim=True) + 1e-5).sqrt() * w1 + b1
        s = r + 0.7 * g * u
        y = s / (s.square().mean(1, keepdim=True) + 1e-5).sqrt() * w2
        return float((s * d(ds)).sum() + (y * d(dy)).sum())

    for k, grad in enumerate([got[0], got[1], got[2], got[3], got[4], got[5]]):
        e = torch.randn(base[k].shape, generator=torch.Generator().manual_seed(k)).double()
        step = 1e-5
        up, down = [[t + (sign * step * e if i == k else 0) for i, t in enumerate(base)] for sign in (1, -1)]
        slope = (value(*up) - value(*down)) / (2 * step)
        # differences: step^2 times third derivatives (below 1e-7 of the sizes here); the gradient: below 1e-4 of its terms
        assert abs(slope - float((d(grad) * e).sum())) <= 1e-5 * float((d(grad) * e).abs().sum()), k


def test_rows_do_not_touch_each_other(fl):
    """A row of NaN, one of infinities and one of zeros: the others' outputs keep their bits."""
    import torch
    h, r, g, c = make(9, 300, "bfloat16", 0, "rms", "layer", "rows", True, "float32", seed=0)
    s, y, _ = fl.fb_residual_norm(h, r, g, want_stats=True, **c)
    bad = h.clone()
    bad[2], bad[5], bad[7] = math.nan, math.inf, 0
    s2, y2 = fl.fb_residual_norm(bad, r, g, **c)
    keep = torch.tensor([0, 1, 3, 4, 6, 8]).cuda()
    assert torch.equal(s[keep], s2[keep]) and torch.equal(y[keep], y2[keep])
    assert s2[2].isnan().all() and y2[2].isnan().all() and y2[5].isnan().all()
    assert torch.equal(s2[7], r[7])                      # the norm of nothing is 0 (eps)


def test_no_rows_and_wanted_outputs(fl):
    import torch
    h, r, g, c = make(0, 33, "float32", 0, "layer", "layer", "vector", True, "float32", seed=3)
    s, y, stats = fl.fb_residual_norm(h, r, g, want_stats=True, **c)
    assert s.shape == y.shape == (0, 33) and stats.shape == (4, 0)
    c.pop("bias", None)
    got = fl.fb_residual_norm_grad(s, y, h, s, stats, g, **c)
    assert got[0].shape == (0, 33) and all(float(t.abs().sum()) == 0 and t.shape == (33,) for t in got[2:])
    h, r, g, c = make(50, 33, "float32", 0, "layer", "layer", "vector", True, "float32", seed=3)
    s, y, stats = fl.fb_residual_norm(h, r, g, want_stats=True, **c)
    c.pop("bias", None)
    full = fl.fb_residual_norm_grad(s, y, h, s, stats, g, **c)
    names = ["want_dh", "want_dresidual", "want_dgate", "want_dinner", "want_douter"]
    index = [(0,), (1,), (2,), (3, 4), (5, 6)]
    for i in range(5):
        some = fl.fb_residual_norm_grad(s, y, h, s, stats, g, **c, **{n: j == i for j, n in enumerate(names)})
        for k in range(7):
            assert (some[k] is not None) == (k in index[i])
            assert some[k] is None or torch.equal(some[k], full[k])


@pytest.mark.parametrize("H", [40, 1000, 3000, 8000])
def test_outputs_in_place_of_inputs(fl, H):
    """Through the C call: s where the residual is and y where h is; the gradients where ds, dy and the gate are."""
    import torch
    import paper_2112_00709_amd as base
    R = 700
    h, r, g, c = make(R, H, "bfloat16", 0, "rms", "layer", "rows", True, "float32", seed=0)
    s, y, stats = fl.fb_residual_norm(h, r, g, want_stats=True, **c)
    w1, w2, b2 = [None if c.get(k) is None else c[k].data_ptr() for k in ("inner_weight", "weight", "bias")]
    st = torch.cuda.current_stream().cuda_stream
    hh, rr = h.clone(), r.clone()
    base._check(fl.lib().fb_residual_norm(hh.data_ptr(), H, rr.data_ptr(), H, g.data_ptr(), H, 0.7, 2, w1, None, 1, w2, b2, 0, R, H, 1, 1e-5,
                                          rr.data_ptr(), H, hh.data_ptr(), H, None, st))
    assert torch.equal(rr, s) and torch.equal(hh, y)
    ds, dy = rows(R, H, "bfloat16", 0, 8), rows(R, H, "bfloat16", 0, 9)
    c.pop("bias", None)
    want = fl.fb_residual_norm_grad(ds, dy, h, s, stats, g, **c, want_dinner=False, want_douter=False)
    gg = g.clone()
    base._check(fl.lib().fb_residual_norm_grad(ds.data_ptr(), H, dy.data_ptr(), H, h.data_ptr(), H, s.data_ptr(), H, stats.data_ptr(), gg.data_ptr(), H, 0.7, 2,
                                               w1, None, 1, w2, 0, R, H, 1, dy.data_ptr(), H, ds.data_ptr(), H, gg.data_ptr(), H, None, None, None, None,
                                               None, 0, st))
    assert torch.equal(dy, want[0]) and torch.equal(ds, want[1]) and torch.equal(gg, want[2])


def test_rows_far_apart(fl):
    """Offsets beyond 2^32 elements."""
    import torch
    R, H, ld = 4200, 64, 1 << 20
    big = torch.empty(R * ld, dtype=torch.bfloat16, device="cuda")
    h = big.as_strided((R, H), (ld, 1))
    src = rows(R, H, "bfloat16", 0, 1)
    h.copy_(src)
    s, y = fl.fb_residual_norm(h, src, outer="rms", inner="layer")
    s2, y2 = fl.fb_residual_norm(src, src, outer="rms", inner="layer")
    assert torch.equal(s, s2) and torch.equal(y, y2)


def test_leading_dimensions_and_single_rows(fl):
    import torch
    h, r, g, c = make(24, 50, "float32", 0, "rms", "rms", "vector", True, "float32", seed=0)
    s, y, stats = fl.fb_residual_norm(h, r, g, want_stats=True, **c)
    s3, y3, st3 = fl.fb_residual_norm(h.view(4, 6, 50), r.view(4, 6, 50), g, want_stats=True, **c)
    assert s3.shape == (4, 6, 50) and st3.shape == (4, 4, 6) and torch.equal(s3.view(24, 50), s) and torch.equal(y3.view(24, 50), y) and torch.equal(st3.view(4, 24), stats)
    s1, y1 = fl.fb_residual_norm(h[3], r[3], g, **c)
    assert torch.equal(s1, s[3]) and torch.equal(y1, y[3])


def test_a_graph_replays_it(fl):
    import torch
    h, r, g, c = make(333, 700, "bfloat16", 0, "layer", "rms", "vector", True, "float32", seed=3)
    ds, dy = rows(333, 700, "bfloat16", 0, 8), rows(333, 700, "bfloat16", 0, 9)
    cg = {k: v for k, v in c.items() if k != "bias"}

    def step():
        s, y, stats = fl.fb_residual_norm(h, r, g, want_stats=True, **c)
        return (s, y, stats, *fl.fb_residual_norm_grad(ds, dy, h, s, stats, g, **cg))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for k in range(3):
        h.copy_(rows(333, 700, "bfloat16", 0, 20 + k))
        want = step()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_refusals(fl):
    import torch
    h = rows(4, 32, "bfloat16", 0, 1)
    w = vector(32, "float32", 2, 1, 0)
    for bad in [dict(inner="rm"), dict(outer="none", weight=w), dict(inner_weight=w), dict(weight=w.half()), dict(weight=w[:31]), dict(residual=h[:3]),
                dict(residual=h.float()), dict(gate=w[:31]), dict(gate=h[:, :16]), dict(gate=w.half()), dict(weight=w, bias=w.bfloat16()),
                dict(gate=w.bfloat16(), weight=w), dict(residual=h.cpu()), dict(gate=h[:1].expand(4, 32)), dict(residual=h.t().contiguous().t())]:
        with pytest.raises(ValueError):
            fl.fb_residual_norm(h, **bad)
    with pytest.raises(ValueError):
        fl.fb_residual_norm(h.long())
    with pytest.raises(fl.FBError) as err:
        fl.fb_residual_norm(rows(2, 8193, "bfloat16", 0, 1))
    assert "8192" in str(err.value)
    for bad in [dict(eps=-1.0), dict(eps=math.nan), dict(scale=math.inf)]:
        with pytest.raises(fl.FBError):
            fl.fb_residual_norm(h, **bad)
    s, y, stats = fl.fb_residual_norm(h, want_stats=True)
    for bad in [dict(dy=None), dict(s=s[:3]), dict(s=s.float()), dict(stats=stats[:3]), dict(dy=y.float()), dict(ds=y[:, :8])]:
        with pytest.raises(ValueError):
            fl.fb_residual_norm_grad(**{**dict(ds=h, dy=y, h=h, s=s, stats=stats), **bad})
    with pytest.raises(ValueError):
        fl.fb_residual_norm_grad(None, None, h, s, stats, outer="none")
