"""Log probabilities of given tokens, entropy, alternatives and their gradient on the GPU against the definition in 64 bits.

Tolerances.  u = 2^-24.  log Z = m + log S: S has terms in (0, 1], the largest 1, each with the error of an exponential of a
rounded argument (e^d (1 + 2 u |d|), |d| e^d <= 0.37, and the exponential's own 2 u) and at most n = V / 64 + 24 roundings of sums
one after the other (wave tree and chunks; far fewer in fact): (n + 4) u relative.  log and the two additions add u each of
max(|m|, |log Z|) .  The entropy's sum of e^d |d| has the same relative error and d an absolute one of u max|x|."""
from __future__ import annotations

import math

import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
H_OF = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}


@pytest.fixture(scope="module")
def fl():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_2112_00709_amd as base
    from paper_2112_00709_amd import layers
    layers.lib()
    base.POISON_NEW_BUFFERS = True
    return layers


def make(R, V, dtype, gap, seed, scale=3.0):
    import torch
    g = torch.Generator().manual_seed(seed)
    x = scale * torch.randn((R, V + gap), generator=g)
    if V > 2:
        x[torch.rand((R, V + gap), generator=g) < 0.05] = -math.inf
    tokens = torch.randint(0, V, (R,), generator=g, dtype=torch.int32)
    if R > 4:
        tokens[1] = -1
        x[1] = math.nan                       # a padded frame holds anything
        x[3] = -math.inf                      # nothing is possible
        x[4, : V] = 0.5                       # everything is as likely
    return x.to(getattr(torch, dtype)).cuda()[:, :V], tokens.cuda()


def definition(x, tokens, top):
    import torch
    xd = x.double().cpu()
    t = tokens.cpu().long()
    R, V = xd.shape
    lp, ent, z = torch.zeros(R, dtype=torch.float64), torch.zeros(R, dtype=torch.float64), torch.zeros(R, dtype=torch.float64)
    ids, best = torch.full((R, top), -1, dtype=torch.int64), torch.zeros((R, top), dtype=torch.float64)
    for r in range(R):
        if t[r] < 0:
            continue
        row = xd[r]
        order = sorted(range(V), key=lambda j: (-row[j].item(), j))[:top] if top else []
        if (row == -math.inf).all():
            z[r] = lp[r] = -math.inf
            ids[r], best[r] = torch.tensor(order), -math.inf
            continue
        z[r] = torch.logsumexp(row, 0)
        logp = row - z[r]
        p = logp.exp()
        lp[r] = logp[t[r]]
        ent[r] = -(p[p > 0] * logp[p > 0]).sum()
        ids[r] = torch.tensor(order, dtype=torch.int64)
        best[r] = logp[ids[r]]
    return lp, ent, z, ids, best


def check(fl, x, tokens, top):
    import torch
    V = x.shape[-1]
    lp, ent, z, ids, best = (t.cpu() for t in fl.fb_token_logprobs(x, tokens, top=top))
    want = definition(x, tokens, top)
    big = torch.where(torch.isfinite(x.double().cpu()), x.double().cpu().abs(), 0.0).amax(1)
    n = V / 64 + 28
    e_z = n * U + 3 * U * (big + math.log(V) + 1)
    for got, ref, e in ((z, want[2], e_z), (lp, want[0], e_z + 2 * U * (2 * big + math.log(V) + 1)), (ent, want[1], 2 * e_z + 2 * n * U * (math.log(V) + 1) + 4 * U * big)):
        got = got.double()
        same = (got == ref) | ((got - ref).abs() <= e)
        assert same.all(), (got[~same], ref[~same])
    assert torch.equal(ids.long(), want[3])
    if top:
        got = best.double()
        same = (got == want[4]) | ((got - want[4]).abs() <= (e_z + 2 * U * (2 * big + math.log(V) + 1))[:, None])
        assert same.all()


@pytest.mark.parametrize("R,V", [(1, 1), (6, 1), (5, 2), (7, 3), (9, 64), (6, 97), (33, 256), (6, 511), (7, 1025), (6, 2050), (5, 4097), (1, 9001),
                                 (2, 33000), (6, 70001), (1, 131072), (1, 300007)])
@pytest.mark.parametrize("dtype,gap", [("float32", 0), ("bfloat16", 5), ("float16", 1)])
def test_against_the_definition(fl, R, V, dtype, gap):
    x, tokens = make(R, V, dtype, gap, R + V)
    for top in sorted({0, 1, min(5, V), min(20, V), min(64, V)}):
        check(fl, x, tokens, top)


@pytest.mark.parametrize("V", [84, 700, 1500, 3000, 4096])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_a_wave_a_row(fl, V, dtype):
    """Enough rows for one wave each; the padded and empty rows are among them."""
    import torch
    x, tokens = make(1100, V, dtype, 1, V)
    lp, ent, z, ids, best = fl.fb_token_logprobs(x, tokens, top=7)
    some = torch.arange(0, 1100, 61)
    some = torch.cat([torch.arange(6), some]).unique()
    few = (x[some.cuda()].contiguous(), tokens[some.cuda()].contiguous())
    check(fl, *few, 7)                             # (fewer rows: perhaps another kernel)
    want = definition(*few, 7)
    assert torch.equal(ids.cpu()[some].long(), want[3])
    got = z.double().cpu()[some]
    assert ((got == want[2]) | ((got - want[2]).abs() <= (V / 64 + 28) * U + 3 * U * (40 + math.log(V)))).all()
    live = (tokens >= 0).cpu()
    assert (ids.cpu()[~live] == -1).all() and (lp.cpu()[~live] == 0).all() and (best.cpu()[~live] == 0).all() and (ent.cpu()[~live] == 0).all()


def test_ties_and_signed_zeros_go_to_the_lowest_number(fl):
    import torch
    for V in (70, 1000, 5000, 40000):
        x = torch.zeros((2, V), device="cuda")
        x[0, ::2] = -0.0                           # equal to 0
        x[1] = torch.arange(V, device="cuda").remainder(5).float()
        ids = fl.fb_token_logprobs(x, torch.zeros(2, dtype=torch.int32, device="cuda"), top=20)[3].cpu()
        assert ids[0].tolist() == list(range(20))
        want = sorted(range(V), key=lambda j: (-(j % 5), j))[:20]
        assert ids[1].tolist() == want


def test_one_lane_holds_all_the_best(fl):
    """Large logits next to each other, and in places 64 vectors apart: more than a wave's lanes can tell apart."""
    import torch
    for V, step in ((4096, 1), (4096, 256), (120000, 2048), (120000, 1)):
        x = torch.randn((3, V), device="cuda", dtype=torch.float32)
        at = torch.arange(0, V, step, device="cuda")[:60]
        x[1, at] += 30 + torch.arange(len(at), device="cuda").float()
        tokens = torch.full((3,), V - 1, dtype=torch.int32, device="cuda")
        check(fl, x, tokens, min(64, V))
        check(fl, x.bfloat16(), tokens, 12)


@pytest.mark.parametrize("V", [40, 106, 300, 512, 513, 2000, 12544, 70001])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_rows_with_few_alternatives(fl, V, dtype):
    """Fewer elements above -inf than alternatives are asked for (0, 1, 3, 30 of them, at the ends and in between): the others
    follow in order of their numbers; and rows of a few values only, many times over."""
    import torch
    x = torch.full((7, V), -math.inf)
    x[1, V - 1] = 2.0
    x[2, [0, V // 2, V - 1]] = torch.tensor([1.0, 1.0, 3.0])
    x[3, torch.arange(0, V, max(1, V // 30))[:30]] = torch.arange(30).float()[: len(torch.arange(0, V, max(1, V // 30))[:30])]
    x[4] = 1.0
    x[5] = torch.arange(V).remainder(3).float()
    x[6, : V // 2] = -1.0
    tokens = torch.full((7,), V - 1, dtype=torch.int32, device="cuda")
    for top in (1, 5, 20, min(64, V)):
        check(fl, x.to(getattr(torch, dtype)).cuda(), tokens, top)


def test_lowest_value_and_large_values(fl):
    """Masks of the type's lowest value instead of -inf; logits near the type's largest."""
    import torch
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        low, high = torch.finfo(dtype).min, torch.finfo(dtype).max
        x = torch.full((3, 130), low, dtype=dtype, device="cuda")
        x[1, 7] = 1.0
        x[2] = high
        tokens = torch.tensor([5, 7, 129], dtype=torch.int32, device="cuda")
        lp, ent, z, ids, best = (t.cpu() for t in fl.fb_token_logprobs(x, tokens, top=3))
        assert abs(ent[0] - math.log(130)) <= 1e-5 and abs(ent[1]) <= 1e-6 and abs(ent[2] - math.log(130)) <= 1e-5
        assert lp[1] == 0 and z[1] == 1.0 and ids[1].tolist() == [7, 0, 1] and ids[0].tolist() == [0, 1, 2]
        assert (x[0, 5].float().cpu() - z[0] == lp[0])


def test_rows_with_nan_or_inf_say_so(fl):
    import torch
    for V in (50, 3000, 60000):
        x = torch.randn((4, V), device="cuda")
        x[1, V // 2] = math.nan
        x[2, V // 3] = math.inf
        tokens = torch.zeros(4, dtype=torch.int32, device="cuda")
        tokens[3] = V                              # no such token
        lp, ent, z, ids, best = (t.cpu() for t in fl.fb_token_logprobs(x, tokens, top=4))
        assert torch.isnan(z[1:3]).all() and torch.isnan(ent[1:3]).all() and torch.isnan(lp[1:]).all()
        assert torch.isfinite(z[[0, 3]]).all() and torch.isfinite(lp[0])


def grad_definition(x, tokens, logz, entropy, g, h):
    import torch
    xd, z, e = x.double().cpu(), logz.double().cpu(), entropy.double().cpu()
    out = torch.zeros_like(xd)
    for r in range(xd.shape[0]):
        if tokens[r] < 0 or z[r] == -math.inf:
            continue
        lp = xd[r] - z[r]
        p = lp.exp()
        out[r] = -p * g[r].double().cpu() - torch.where(p > 0, p * (torch.where(p > 0, lp, 0.0) + e[r]), 0.0) * (h[r].double().cpu() if h is not None else 0.0)
        if tokens[r] < xd.shape[1]:
            out[r, tokens[r]] += g[r].double().cpu()
    return out


@pytest.mark.parametrize("R,V", [(1, 1), (6, 2), (5, 63), (300, 84), (7, 1025), (6, 4099), (2, 70001)])
@pytest.mark.parametrize("dtype,gap", [("float32", 3), ("bfloat16", 0), ("float16", 7)])
def test_gradient_against_the_formula(fl, R, V, dtype, gap):
    import torch
    x, tokens = make(R, V, dtype, gap, 7 * R + V)
    gen = torch.Generator().manual_seed(R)
    g, h = torch.randn(R, generator=gen).cuda(), torch.randn(R, generator=gen).cuda()
    lp, ent, z, _, _ = fl.fb_token_logprobs(x, tokens)
    for gh in ((g, None), (g, h), (None, h)):
        d = fl.fb_token_logprobs_grad(x, tokens, z, ent, *gh)
        gg = gh[0] if gh[0] is not None else torch.zeros_like(g)
        want = grad_definition(x, tokens, z, ent, gg, gh[1])
        # the exponential's argument is rounded at the size of the logits: relative (2 |lp| + 4) u of p, with |lp| p <= 0.37;
        # the entropy's bracket adds u (|lp| + H) p
        size = gg.abs().cpu().double() + (gh[1].abs().cpu().double() * (2 + 2 * math.log(V + 1)) if gh[1] is not None else 0)
        tol = 60 * U * size[:, None] + H_OF[dtype] * want.abs() + (2.0 ** -24 if dtype == "float16" else 0)
        assert ((d.double().cpu() - want).abs() <= tol).all()
        assert d.dtype == x.dtype


@pytest.mark.parametrize("V", [5, 31, 32, 33, 64, 65, 127, 128, 129, 136, 137, 200, 255, 256, 257, 263, 383, 511, 512, 1000, 1025])
@pytest.mark.parametrize("dtype,gap", [("float32", 1), ("bfloat16", 0), ("float16", 3)])
def test_short_rows_of_every_kind_of_end(fl, V, dtype, gap):
    """Rows that end inside, at and after a piece of 16 bytes, as many as do not fill a workgroup; few and many alternatives."""
    import torch
    R = 37
    x, tokens = make(R, V, dtype, gap, V)
    tokens[5], tokens[6] = V - 1, 0
    for top in sorted({min(t, V) for t in (0, 3, 24, 25)}):
        check(fl, x, tokens, top)
    gen = torch.Generator().manual_seed(V)
    g, h = torch.randn(R, generator=gen).cuda(), torch.randn(R, generator=gen).cuda()
    lp, ent, z, _, _ = fl.fb_token_logprobs(x, tokens)
    d = fl.fb_token_logprobs_grad(x, tokens, z, ent, g, h)
    want = grad_definition(x, tokens, z, ent, g, h)
    size = g.abs().cpu().double() + h.abs().cpu().double() * (2 + 2 * math.log(V + 1))
    tol = 60 * U * size[:, None] + H_OF[dtype] * want.abs() + (2.0 ** -24 if dtype == "float16" else 0)
    assert ((d.double().cpu() - want).abs() <= tol).all()


def test_gradient_against_differences(fl):
    import torch
    gen = torch.Generator().manual_seed(3)
    x = torch.randn((2, 11), generator=gen)
    tokens = torch.tensor([4, 10], dtype=torch.int32)
    g, h = torch.tensor([0.7, -1.2]), torch.tensor([0.4, 0.9])
    lp, ent, z, _, _ = fl.fb_token_logprobs(x.cuda(), tokens.cuda())
    d = fl.fb_token_logprobs_grad(x.cuda(), tokens.cuda(), z, ent, g.cuda(), h.cuda()).cpu().double()

    def f(x):
        l, e, _, _, _ = definition(x, tokens, 0)
        return float((l * g.double()).sum() + (e * h.double()).sum())

    x = x.double()
    step = 1e-5
    for r in range(2):
        for j in range(11):
            keep = x[r, j].item()
            x[r, j] = keep + step
            up = f(x)
            x[r, j] = keep - step
            down = f(x)
            x[r, j] = keep
            assert abs((up - down) / (2 * step) - d[r, j].item()) <= 2e-6


def test_no_rows_leading_shapes_and_another_stream(fl):
    import torch
    x = torch.empty((0, 9), device="cuda")
    t = torch.empty((0,), dtype=torch.int32, device="cuda")
    out = fl.fb_token_logprobs(x, t, top=2)
    assert out[0].shape == (0,) and out[3].shape == (0, 2)
    assert fl.fb_token_logprobs_grad(x, t, out[2], out[1], out[0]).shape == (0, 9)
    x, tokens = make(12, 9000, "bfloat16", 0, 2)
    flat = fl.fb_token_logprobs(x, tokens, top=3)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = fl.fb_token_logprobs(x.view(3, 4, 9000), tokens.view(3, 4), top=3)
    s.synchronize()
    for a, b in zip(flat, other):
        assert torch.equal(a, b.view(a.shape)) or (torch.isnan(a) == torch.isnan(b.view(a.shape))).all()


def test_more_rows_than_a_launch_takes(fl):
    """Rows beyond the first 2^22, and beyond 2^24 pieces of the gradient: the last ones are as the first."""
    import torch
    R = (1 << 24) + 77
    g = torch.Generator().manual_seed(5)
    few = torch.randn((64, 3), generator=g).cuda()
    x = few.repeat((R + 63) // 64, 1)[:R].contiguous()
    tokens = torch.arange(R, dtype=torch.int32, device="cuda") % 3
    lp, ent, z, ids, _ = fl.fb_token_logprobs(x, tokens, top=2)
    d = fl.fb_token_logprobs_grad(x, tokens, z, ent, torch.ones(R, device="cuda"), ent)
    head = fl.fb_token_logprobs(x[-100:].contiguous(), tokens[-100:].contiguous(), top=2)
    for a, b in zip((lp, ent, z, ids), head):
        assert torch.equal(a[-100:], b)
    dh = fl.fb_token_logprobs_grad(x[-100:].contiguous(), tokens[-100:].contiguous(), head[2], head[1], torch.ones(100, device="cuda"), head[1])
    assert torch.equal(d[-100:], dh)
    assert torch.isfinite(lp).all() and torch.isfinite(d).all()


def test_recorded_into_a_graph(fl):
    import torch
    x, tokens = make(3, 50000, "bfloat16", 0, 21)
    g = torch.ones(3, device="cuda")

    def step():
        out = fl.fb_token_logprobs(x, tokens, top=6)
        return (*out, fl.fb_token_logprobs_grad(x, tokens, out[2], out[1], g, g))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for seed in (22, 23, 24):
        x.copy_(make(3, 50000, "bfloat16", 0, seed)[0])
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, step()):
            assert torch.equal(a, b)


def test_refusals(fl):
    import torch
    x, t = torch.zeros((4, 8), device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        fl.fb_token_logprobs(x, t.long())
    with pytest.raises(ValueError):
        fl.fb_token_logprobs(x, t[:3])
    with pytest.raises(ValueError):
        fl.fb_token_logprobs(x.double(), t)
    with pytest.raises(ValueError):
        fl.fb_token_logprobs(x.cpu(), t)
    for top in (-1, 9, 65):
        with pytest.raises((fl.FBError, RuntimeError)):
            fl.fb_token_logprobs(x, t, top=top)
    with pytest.raises(fl.FBError):
        fl.fb_token_logprobs_grad(x, t, t.float(), None, t.float(), t.float())   # entropy's gradient without the entropy
    with pytest.raises(ValueError):
        fl.fb_token_logprobs_grad(x, t, t.float()[:3], t.float(), t.float())
