"""Log probabilities and entropy straight from hidden frames, and their gradient, on the GPU against the definitions in 64 bits.

Tolerances.  u = 2^-24, h the type's roundoff.  A logit is a sum of K + 1 terms, formed with at most K + 16 roundings: off by at most
e = 2 (K + 16) u (sum |x w| + |bias|).  S = sum e^(z - m) is off by e in every term, by the roundings of the exponents, 8 u |z| at most,
and by those of the sums, 400 + V / 64 at most one after the other: r = 8 u max |z| + (400 + V / 64) u, relative.  So
log Z is off by max e + r + 2 u |log Z| and a log probability by e more.  The entropy's derivative with respect to a logit is
-p (log p + E), whose sizes add up to 2 E at most: 2 E (max e + r) + 2 r + 4 u (1 + E + log V).
dz = g [j = token] - p (a + h log p):  p is off by f = e + u (4 |z| + 4 |log Z| + 8) of its size, log p by f: dz by
p (f (|a| + |h| |log p| + |h|) + 8 u (|g| + |h| |E| + |h log p|)) + u |dz|.  It is rounded once before the products where the type has 16 bits,
in half precision with at least 2^-38 of the largest bound of |dz|; the products are off by 2 (300 + n / 8) u of their terms' sizes, and the
outputs are rounded once."""
from __future__ import annotations

import math

import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
H_OF = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
TINY = {"float32": 1e-37, "bfloat16": 1e-37, "float16": 2.0 ** -24}
TYPES = [("float32", 0), ("bfloat16", 0), ("float16", 3), ("bfloat16", 8)]
SIZES = [(1, 1, 1), (1, 40, 33), (1, 128000, 64), (2, 17, 1), (16, 3000, 1024), (17, 1000, 72), (33, 700, 130), (64, 5001, 40), (48, 84, 4096), (64, 70001, 16),
         (65, 1, 16), (65, 2, 24), (66, 257, 129), (100, 40000, 40), (200, 84, 1024), (257, 3000, 200), (1000, 1500, 264), (513, 2555, 777), (3000, 20, 520),
         (2600, 8200, 72), (9000, 2050, 40)]


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


def numbers(n, seed, scale=1.0):
    return rows(1, n, "float32", 0, seed, scale)[0]


def inputs(M, V, K, dtype, gap, seed, pad=0.2, out=0.1):
    """x, weight, bias, tokens; some rows do not count, with NaN in x, and some alternatives are ruled out (never the first)."""
    import torch
    g = torch.Generator().manual_seed(seed)
    x, w, b = rows(M, K, dtype, gap, seed + 1), rows(V, K, dtype, gap and 8, seed + 2, 2 * K ** -0.5), numbers(V, seed + 3)
    tokens = torch.randint(0, V, (M,), generator=g, dtype=torch.int32)
    none = torch.rand(M, generator=g) < pad if M > 1 else torch.zeros(M, dtype=torch.bool)
    tokens[none] = torch.where(torch.arange(int(none.sum())) % 2 == 0, -1, -2 ** 31).to(torch.int32)
    x[none.cuda()] = math.nan
    ruled = torch.rand(V, generator=g) < out
    ruled[0] = False
    b[ruled.cuda()] = -math.inf
    return x, w, b, tokens.cuda()


def logits_of(x, w, b, tokens):
    """-> logits in 64 bits and how far they may be off."""
    live = (tokens >= 0)[:, None]
    x = x.double().masked_fill(~live, 0)
    w = w.double().contiguous()
    z, e = x @ w.t().contiguous(), x.abs() @ w.abs().t().contiguous()
    if b is not None:
        z, e = z + b.double(), e + b.double().abs().masked_fill(b == -math.inf, 0)
    return z, 2 * (x.shape[1] + 16) * U * e


def close(got, want, tol, dtype, what):
    import torch
    got = got.double()
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    bad = ~same & ~((got - want).abs() <= tol + H_OF[dtype] * (want.abs() + tol) * 1.01 + TINY[dtype])
    assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[:4].tolist(), got[bad][:4], want[bad][:4])


def finite_max(z):
    import torch
    return torch.where(torch.isfinite(z), z.abs(), torch.zeros_like(z)).max(1).values


def check_forward(fl, x, w, b, tokens):
    import torch
    V = w.shape[0]
    lp, ent, logz = fl.fb_affine_logprobs(x, w, tokens, b)
    z, e = logits_of(x, w, b, tokens)
    live = tokens >= 0
    want_z = torch.logsumexp(z, 1)
    p = torch.exp(z - want_z[:, None])
    want_e = -torch.xlogy(p, p).sum(1)
    at = tokens.clamp_min(0).long()[:, None]
    given, e_given = z.gather(1, at)[:, 0], e.gather(1, at)[:, 0]
    off = e.max(1).values
    r = 8 * U * finite_max(z) + (400 + V / 64) * U
    for got, want, tol, what in ((logz, want_z, off + r + 2 * U * want_z.abs(), "logz"),
                                 (lp, given - want_z, e_given + off + r + 4 * U * (given.abs().masked_fill(torch.isinf(given), 0) + want_z.abs()), "logprobs"),
                                 (ent, want_e, 2 * want_e * (off + r) + 2 * r + 4 * U * (1 + want_e + math.log(V)), "entropy")):
        assert got.shape == tokens.shape and got.dtype == torch.float32
        close(got, want.masked_fill(~live, 0), tol, "float32", what)
    return lp, ent, logz


def check_grad(fl, x, w, b, tokens, g, h, forward=None):
    import torch
    dtype = str(x.dtype)[6:]
    (M, K), V = x.shape, w.shape[0]
    _, ent, logz = forward or fl.fb_affine_logprobs(x, w, tokens, b)
    got = fl.fb_affine_logprobs_grad(x, w, tokens, logz, None if h is None else ent, g, h, b)
    z, e = logits_of(x, w, b, tokens)
    live = (tokens >= 0)[:, None]
    lz, en = logz.double()[:, None], ent.double()[:, None]
    gd = torch.zeros_like(lz) if g is None else g.double()[:, None]
    hd = torch.zeros_like(lz) if h is None else h.double()[:, None]
    logp = (z - lz).clamp_min(-1e4)
    p = torch.exp(logp)
    a = gd + hd * en
    dz = -p * (a + hd * logp)
    f = e + U * (4 * z.abs().masked_fill(torch.isinf(z), 0) + 4 * lz.abs() + 8)
    off = p * (f * (a.abs() + hd.abs() * logp.abs() + hd.abs()) + 8 * U * (gd.abs() + (hd * en).abs() + (hd * logp).abs()))
    at = tokens.clamp(0, V - 1).long()[:, None]
    dz.scatter_add_(1, at, torch.where(live & (tokens < V)[:, None], gd, 0))
    off = (off + U * dz.abs()).masked_fill(~live, 0)
    dz = dz.masked_fill(~live, 0)
    close(got[2], dz.sum(0), (300 + M / 16) * U * dz.abs().sum(0) + off.sum(0), "float32", "dbias")
    if dtype != "float32":
        off = off + H_OF[dtype] * 1.01 * dz.abs()
    if dtype == "float16":
        off = off + float((gd.abs() + hd.abs() * (0.37 + en.abs())).max()) * 2.0 ** -38
    xd, wd = x.double().masked_fill(~live, 0), w.double().contiguous()
    size = dz.abs()
    close(got[0], dz @ wd, 1.01 * (2 * (300 + V / 8) * U * (size @ wd.abs()) + off @ wd.abs()), dtype, "dx")
    back = 1.01 * (2 * (300 + M / 16) * U * (size.t().contiguous() @ xd.abs()) + off.t().contiguous() @ xd.abs())
    close(got[1], dz.t().contiguous() @ xd, back, dtype, "dweight")
    assert got[0].dtype == x.dtype and got[1].dtype == w.dtype and got[2].dtype == torch.float32
    assert not got[0][tokens < 0].any()
    return got


@pytest.mark.parametrize("M,V,K", SIZES)
@pytest.mark.parametrize("dtype,gap", TYPES)
def test_forward(fl, M, V, K, dtype, gap):
    x, w, b, tokens = inputs(M, V, K, dtype, gap, M + V + K)
    check_forward(fl, x, w, b, tokens)
    check_forward(fl, x, w, None, tokens)


@pytest.mark.parametrize("M,V,K", SIZES)
@pytest.mark.parametrize("dtype,gap", TYPES)
def test_gradient(fl, M, V, K, dtype, gap):
    x, w, b, tokens = inputs(M, V, K, dtype, gap, M + V + K)
    g, h = numbers(M, 5), numbers(M, 6, 0.1)
    forward = fl.fb_affine_logprobs(x, w, tokens, b)
    check_grad(fl, x, w, b, tokens, g, h, forward)
    check_grad(fl, x, w, b, tokens, g, None, forward)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_a_vocabulary_in_pieces(fl, dtype):
    """The logits' gradient would take more than half a gigabyte: pieces add up, tokens of all of them, the last shorter."""
    M, V, K = (1100, 131011, 24) if dtype == "float32" else (2200, 131011, 24)
    x, w, b, tokens = inputs(M, V, K, dtype, 3, 7)
    tokens[:6] = fl.torch.tensor([0, V - 1, 65535, 65536, V // 2, 131010])
    x[:6] = 1.0
    b[tokens[:6].long()] = 0.5
    got = check_grad(fl, x, w, b, tokens, numbers(M, 5), numbers(M, 6, 0.1))
    _, ent, logz = fl.fb_affine_logprobs(x, w, tokens, b)
    again = fl.fb_affine_logprobs_grad(x, w, tokens, logz, ent, numbers(M, 5), numbers(M, 6, 0.1), b)
    for p, q in zip(got, again):
        assert fl.torch.equal(p, q)


@pytest.mark.parametrize("M,V,K", [(3, 300, 40), (300, 700, 72)])
@pytest.mark.parametrize("size", [1e-7, 1e-3, 3e4])
def test_half_precision_gradients_of_any_size(fl, M, V, K, size):
    x, w, b, tokens = inputs(M, V, K, "float16", 0, 3)
    w = w * 0.01 if size > 1 else w
    x = x * 0.01 if size > 1 else x
    check_grad(fl, x, w, b, tokens, numbers(M, 5, size).abs().clamp(0, size), numbers(M, 6, size * 0.1))


@pytest.mark.parametrize("M,V,K", [(5, 700, 72), (64, 40, 40), (300, 700, 72), (2600, 2050, 40)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_rows_of_nothing_and_broken_rows(fl, M, V, K, dtype):
    """All alternatives ruled out; NaN and infinities in a row of x; tokens past the vocabulary."""
    import torch
    x, w, b, tokens = inputs(M, V, K, dtype, 0, 11, pad=0.0, out=0.0)
    g, h = numbers(M, 5), numbers(M, 6)
    for low in (-math.inf, torch.finfo(torch.float32).min):
        lp, ent, logz = fl.fb_affine_logprobs(x, w, tokens, torch.full_like(b, low))
        assert (lp == -math.inf).all() and (logz == -math.inf).all() and not ent.any()
        broken = x.clone()
        broken[1] = math.inf                                # (nothing of such a row counts)
        for t in fl.fb_affine_logprobs_grad(broken, w, tokens, logz, ent, g, h, torch.full_like(b, low)):
            assert not t.any() and not torch.isnan(t).any()
    one = torch.full_like(b, -math.inf)
    one[V // 3] = -5.0                                      # a single alternative left: log Z is its logit, and nothing to decide
    lp, ent, logz = check_forward(fl, x, w, one, tokens)
    assert (ent.abs() < 1e-5).all()
    tokens[2] = V
    tokens[3] = 2 ** 31 - 1
    lp, ent, logz = fl.fb_affine_logprobs(x, w, tokens, b)
    past = tokens >= V
    assert torch.isnan(lp[past]).all() and not torch.isnan(lp[~past]).any() and torch.isfinite(ent).all() and torch.isfinite(logz).all()
    check_grad(fl, x, w, b, tokens, g, h)
    for broken in (math.nan, math.inf):
        y = x.clone()
        y[1, K - 1] = broken
        w[:, K - 1] = w[:, K - 1].abs() + 0.25
        out = fl.fb_affine_logprobs(y, w, tokens, b)
        for t in out:
            assert torch.isnan(t[1]) and not torch.isnan(t[4:]).any()
        dx, dw, db = fl.fb_affine_logprobs_grad(y, w, tokens, out[2], out[1], g, h, b)
        assert torch.isnan(dx[1]).all() and torch.isfinite(dx[4:]).all() and torch.isnan(dw).all() and torch.isnan(db).all()


@pytest.mark.parametrize("M", [7, 300])
@pytest.mark.parametrize("shift", [1e4, -1e4, 3e37, -3e37])
def test_large_logits(fl, M, shift):
    """A level that all logits share leaves log probabilities and entropy as they are, to the digits that the logits have."""
    import torch
    x, w, b, tokens = inputs(M, 500, 8, "float32", 0, 21, pad=0.0, out=0.0)
    w = (w * 0).contiguous()
    b = torch.where(torch.arange(500, device="cuda") % 2 == 0, shift, shift - abs(shift) * 2.0 ** -10)
    lp, ent, logz = fl.fb_affine_logprobs(x, w, tokens, b)
    even = tokens % 2 == 0
    far = abs(shift) * 2.0 ** -10                            # 9.8: the others have e^-9.8 of the weight
    rest = math.exp(-far)
    logz_off = math.log(250 * (1 + rest))
    entropy = logz_off + rest * far / (1 + rest) if far < 100 else math.log(250)
    # (log Z rounded to the level's digits: u |shift| each for it and the difference)
    assert ((logz.double() - shift - logz_off).abs() <= 4 * U * abs(shift)).all()
    assert ((ent.double() - entropy).abs() <= 500 * U * 16 + 1e-4).all()
    assert ((lp.double() + logz_off)[even].abs() <= 4 * U * abs(shift) + 1e-4).all()
    assert torch.isfinite(lp).all()


def test_agrees_with_the_calls_that_keep_the_logits(fl):
    """fb_affine into single precision and fb_token_logprobs of its logits: the same definitions, outputs and gradients."""
    import torch
    for M, V, K in [(3, 500, 40), (700, 3000, 264)]:
        x, w, b, tokens = inputs(M, V, K, "float32", 0, 31)
        x = torch.nan_to_num(x)
        logits = fl.fb_affine(x, w, b)
        apart = fl.fb_token_logprobs(logits, tokens)[:3]
        here = fl.fb_affine_logprobs(x, w, tokens, b)
        for p, q in zip(here, apart):
            close(p, q.double(), 1e-5 * (1 + q.double().abs().masked_fill(torch.isinf(q), 0)), "float32", "forward")
        g, h = numbers(M, 5), numbers(M, 6)
        dl = fl.fb_token_logprobs_grad(logits, tokens, apart[2], apart[1], g, h)
        for p, q in zip(fl.fb_affine_logprobs_grad(x, w, tokens, here[2], here[1], g, h, b), fl.fb_affine_grad(dl, x, w)):
            # (logits off by 2 (K + 16) u sum |x w|, up to 2e-3: of dz that much, of sums the terms' sizes, up to 30)
            assert ((p - q).abs() <= 2e-3 * (1 + q.abs())).all()


def test_gradient_against_differences(fl):
    import torch
    gen = torch.Generator().manual_seed(8)
    M, V, K = 4, 7, 5
    x, w, b, cg, ch = (torch.randn(s, generator=gen) for s in ((M, K), (V, K), (V,), (M,), (M,)))
    tokens = torch.tensor([3, -1, 0, 6], dtype=torch.int32)
    _, ent, logz = fl.fb_affine_logprobs(x.cuda(), w.cuda(), tokens.cuda(), b.cuda())
    got = [t.double().cpu() for t in fl.fb_affine_logprobs_grad(x.cuda(), w.cuda(), tokens.cuda(), logz, ent, cg.cuda(), ch.cuda(), b.cuda())]

    def f(x, w, b):
        logp = torch.log_softmax(x @ w.t() + b, 1)
        each = cg.double() * logp.gather(1, tokens.clamp_min(0).long()[:, None])[:, 0] - ch.double() * (logp.exp() * logp).sum(1)
        return float(each[tokens >= 0].sum())

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
            # (differences: step^2 = 1e-10 of third derivatives; single precision: some 100 u = 6e-6 of terms of size 3)
            assert abs((up - down) / (2 * step) - want.reshape(-1)[i].item()) <= 5e-5


@pytest.mark.parametrize("M,V,K,dtype", [(5, 300, 72, "float32"), (700, 3000, 264, "bfloat16"), (400, 555, 77, "float16")])
def test_parts_of_the_gradient(fl, M, V, K, dtype):
    """What is left out leaves the rest as it is; a second call gives the same bits, also on another stream and of other leading shapes."""
    import torch
    x, w, b, tokens = inputs(M, V, K, dtype, 0, 41)
    g, h = numbers(M, 5), numbers(M, 6)
    forward = fl.fb_affine_logprobs(x, w, tokens, b)
    full = fl.fb_affine_logprobs_grad(x, w, tokens, forward[2], forward[1], g, h, b)
    for want in [(True, False, False), (False, True, False), (False, False, True), (True, False, True), (True, True, True), (False, False, False)]:
        got = fl.fb_affine_logprobs_grad(x, w, tokens, forward[2], forward[1], g, h, b, *want)
        for p, q, asked in zip(got, full, want):
            assert (p is None) == (not asked)
            assert not asked or torch.equal(p, q)
    none = fl.fb_affine_logprobs_grad(x, w, tokens, forward[2], None, None, None, b)
    assert not any(t.any() for t in none)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        y, t = x.reshape(1, M, K), tokens.view(1, M)
        other = fl.fb_affine_logprobs(y, w, t, b)
        back = fl.fb_affine_logprobs_grad(y, w, t, other[2], other[1], g.view(1, M), h.view(1, M), b)
    s.synchronize()
    for p, q in zip((*other, *back), (*forward, *full)):
        assert torch.equal(p.view(q.shape), q)


def test_no_rows(fl):
    import torch
    x, w, tokens = torch.empty((0, 30), device="cuda"), rows(40, 30, "float32", 0, 1), torch.empty(0, dtype=torch.int32, device="cuda")
    out = fl.fb_affine_logprobs(x, w, tokens)
    assert all(t.shape == (0,) for t in out)
    dx, dw, db = fl.fb_affine_logprobs_grad(x, w, tokens, out[2], out[1], out[0], None)
    assert dx.shape == (0, 30) and torch.equal(dw, torch.zeros_like(w)) and torch.equal(db, torch.zeros(40, device="cuda"))
    x, tokens = rows(70, 30, "bfloat16", 0, 2), torch.full((70,), -1, dtype=torch.int32, device="cuda")
    w = w.bfloat16()
    out = fl.fb_affine_logprobs(x, w, tokens)
    assert not any(t.any() for t in out)
    for t in fl.fb_affine_logprobs_grad(x, w, tokens, out[2], out[1], out[0] + 1, None):
        assert not t.any() and not torch.isnan(t).any()


@pytest.mark.parametrize("M,V,K,dtype", [(5, 300, 72, "bfloat16"), (700, 3000, 264, "float16"), (1100, 2050, 40, "float32")])
def test_recorded_into_a_graph(fl, M, V, K, dtype):
    import torch
    x, w, b, tokens = inputs(M, V, K, dtype, 0, 51)
    g, h = numbers(M, 5), numbers(M, 6)

    def step():
        out = fl.fb_affine_logprobs(x, w, tokens, b)
        return (*out, *fl.fb_affine_logprobs_grad(x, w, tokens, out[2], out[1], g, h, b))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for seed in (13, 14, 15):
        nx, _, _, nt = inputs(M, V, K, dtype, 0, seed)
        x.copy_(nx)
        tokens.copy_(nt)
        graph.replay()
        torch.cuda.synchronize()
        for p, q in zip(got, step()):
            assert torch.equal(p, q)


def test_offsets_beyond_32_bits(fl):
    """x of more than 2^31 elements and 4 GB, whose last rows count."""
    import torch
    M, V, K = 1_100_000, 40, 2048
    x = torch.zeros((M, K), dtype=torch.bfloat16, device="cuda")
    x[-70:] = rows(70, K, "bfloat16", 0, 1)
    _, w, b, last = inputs(70, V, K, "bfloat16", 0, 2, pad=0.0)
    tokens = torch.full((M,), -1, dtype=torch.int32, device="cuda")
    tokens[-70:] = last
    out = fl.fb_affine_logprobs(x, w, tokens, b)
    few = check_forward(fl, x[-70:].contiguous(), w, b, last)
    assert all(not t[:-70].any() for t in out)
    g = numbers(M, 5)
    dx, dw, db = fl.fb_affine_logprobs_grad(x, w, tokens, out[2], None, g, None, b)
    small = fl.fb_affine_logprobs_grad(x[-70:].contiguous(), w, last, out[2][-70:].contiguous(), None, g[-70:].contiguous(), None, b)
    for t, q in zip(out, few):                               # (tiles of another size: sums in another order, some 1e-6 of numbers up to 20)
        assert ((t[-70:] - q).abs().nan_to_num(0.0) <= 1e-4).all()
    assert not dx[:-70].any()
    for t, q in zip((dx[-70:], dw, db), small):              # (16 bits twice)
        assert ((t.float() - q.float()).abs() <= 2.0 ** -7 * q.float().abs() + 2e-2).all()


def test_refusals(fl):
    import torch
    x, w, b, t = torch.zeros((4, 8), device="cuda"), torch.zeros((6, 8), device="cuda"), torch.zeros(6, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    bad = [dict(x=x.cpu()), dict(x=x.double()), dict(x=x.t()), dict(weight=w[:, :7]), dict(weight=w.bfloat16()), dict(weight=w.view(-1)), dict(weight=w.cpu()),
           dict(tokens=t[:3]), dict(tokens=t.long()), dict(tokens=t.view(2, 2)), dict(tokens=t.cpu()), dict(bias=b[:5]), dict(bias=b.half()), dict(bias=b.cpu())]
    for change in bad:
        with pytest.raises(ValueError):
            fl.fb_affine_logprobs(**{**dict(x=x, weight=w, tokens=t, bias=b), **change})
    z = torch.zeros(4, device="cuda")
    base = dict(x=x, weight=w, tokens=t, logz=z, entropy=z, g_logprobs=z, g_entropy=z, bias=b)
    for change in bad + [dict(logz=z[:3]), dict(logz=z.double()), dict(entropy=z.half()), dict(g_logprobs=z.cpu()), dict(g_entropy=z[:2])]:
        with pytest.raises(ValueError):
            fl.fb_affine_logprobs_grad(**{**base, **change})
    for change in [dict(logz=None), dict(entropy=None)]:
        with pytest.raises(fl.FBError):
            fl.fb_affine_logprobs_grad(**{**base, **change})
    with pytest.raises(ValueError):                          # (rows of no elements cannot be counted)
        fl.fb_affine_logprobs(torch.zeros((4, 0), device="cuda"), torch.zeros((6, 0), device="cuda"), t)
    with pytest.raises(fl.FBError):
        fl.fb_affine_logprobs(x, w[:0], t)
