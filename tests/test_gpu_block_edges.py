"""The block operators at addresses, layouts and in company that their other tests do not have: every operand from an odd element on, two
streams at once, calls on memory that earlier calls left dirty, one element a row."""
from __future__ import annotations

import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fl():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_2112_00709_amd as base
    from paper_2112_00709_amd import layers
    layers.lib()
    base.POISON_NEW_BUFFERS = True
    return layers


def odd(t, off):
    """The same numbers in rows that start `off` elements behind a 16-byte boundary and lie at an odd distance, NaN between them."""
    import torch
    if t.dim() == 1:
        wide = torch.full((t.numel() + 9,), math.nan, device="cuda").to(t.dtype) if t.dtype.is_floating_point else torch.zeros(t.numel() + 9, dtype=t.dtype, device="cuda")
        view = wide[off:off + t.numel()]
    else:
        wide = torch.full((t.shape[0], t.shape[1] + 9 + (t.shape[1] + 9) % 2 - 1), math.nan, device="cuda").to(t.dtype)
        view = wide[:, off:off + t.shape[1]]
    view.copy_(t)
    return view


def same(a, b):
    import torch
    for x, y in zip(a, b):
        assert (x is None) == (y is None)
        if x is not None:
            assert not torch.isnan(x).any() and torch.equal(x, y)


def make(M, N, K, dtype, seed):
    import torch
    g = torch.Generator().manual_seed(seed)
    t = getattr(torch, dtype)

    def r(*shape):
        return torch.randn(shape, generator=g).cuda()

    c = dict(x=r(M, K).to(t), w2=(r(2 * N, K) * K ** -0.5).to(t), wv=(r(N, K) * K ** -0.5).to(t), dy=r(M, N).to(t), z=r(M, 2 * N).to(t), b2=r(2 * N), bv=r(N), g=r(M), h=r(M),
             h0=r(M, K).to(t), res=r(M, K).to(t), gate=r(M, K).to(t), nw=1 + 0.1 * r(K), nb=r(K))
    c["tokens"] = torch.randint(-1, N, (M,), generator=g, dtype=torch.int32).cuda()
    return c


def run(fl, c, seen=None):
    s, y, stats = fl.fb_residual_norm(c["h0"], c["res"], c["gate"], 0.5, "layer", c["nw"], c["nb"], "rms", c["nw"], None, want_stats=True)
    back = fl.fb_residual_norm_grad(c["x"], c["res"], c["h0"], s if seen is None else seen["s"], stats, c["gate"], 0.5, "layer", c["nw"], c["nb"], "rms", c["nw"])
    gated = fl.fb_gated_affine(c["x"], c["w2"], c["b2"], want_preact=True)
    gback = fl.fb_gated_affine_grad(c["dy"], c["x"], c["w2"], c["z"], activation="gelu")
    lp = fl.fb_affine_logprobs(c["x"], c["wv"], c["tokens"], c["bv"])
    lback = fl.fb_affine_logprobs_grad(c["x"], c["wv"], c["tokens"], lp[2], lp[1], c["g"], c["h"], c["bv"])
    return [s, y, stats, *back, *gated, *gback, *lp, *lback]


SIZES = [(1, 7, 33), (5, 40, 8), (64, 130, 72), (65, 66, 40), (300, 257, 136), (1031, 515, 264)]


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("off", [1, 3])
def test_operands_from_any_element_on(fl, M, N, K, dtype, off):
    """The same bits as from aligned, contiguous ones."""
    c = make(M, N, K, dtype, M + N)
    plain = run(fl, c)
    moved = {k: odd(v, off) for k, v in c.items()}
    same(run(fl, moved, seen=dict(s=odd(plain[0], off))), plain)


def test_two_streams_at_once(fl):
    """Calls of different inputs under way at the same time: the bits of each alone."""
    import torch
    cs = [make(1500, 900, 264, "float16", s) for s in (1, 2)]
    alone = [run(fl, c) for c in cs]
    streams = [torch.cuda.Stream() for _ in cs]
    got = [None, None]
    torch.cuda.synchronize()
    for _ in range(3):
        for k in (0, 1):
            with torch.cuda.stream(streams[k]):
                got[k] = run(fl, cs[k])
        torch.cuda.synchronize()
        for a, b in zip(got, alone):
            same(a, b)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_nothing_is_read_that_was_not_written(fl, dtype):
    """Workspaces and outputs hold NaN before every call here (or zeros): the results do not tell."""
    import torch

    import paper_2112_00709_amd as base
    for M, N, K in SIZES:
        c = make(M, N, K, dtype, 3)
        poisoned = run(fl, c)
        base.POISON_NEW_BUFFERS = False
        try:
            torch.cuda.empty_cache()
            same(run(fl, c), poisoned)
        finally:
            base.POISON_NEW_BUFFERS = True


def test_captured_calls_among_eager_ones(fl):
    """Two graphs of different sizes replayed in turn with eager calls between them."""
    import torch
    cs = [make(200, 66, 72, "bfloat16", 5), make(700, 515, 136, "float16", 6)]
    for c in cs:
        run(fl, c)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for c in cs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(run(fl, c))
        graphs.append(graph)
    for turn in range(3):
        for c in cs:
            c["x"].mul_(0.9)
            c["tokens"].copy_(torch.roll(c["tokens"], 1))
        for k in (1, 0):
            graphs[k].replay()
            run(fl, make(300, 40, 40, "float32", turn))
        torch.cuda.synchronize()
        for k in (0, 1):
            same(outs[k], run(fl, cs[k]))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_one_element_a_row(fl, dtype):
    """K = 1, N = 1: a logit among one alternative, a gated layer of one output, norms of one element."""
    import torch
    for M in (1, 65, 300):
        c = make(M, 1, 1, dtype, 7)
        c["tokens"].clamp_(min=0)
        out = run(fl, c)
        assert all(torch.isfinite(t).all() for t in out if t is not None)
        lp, ent, logz = fl.fb_affine_logprobs(c["x"], c["wv"], c["tokens"], c["bv"])
        assert lp.abs().max() <= 1e-5 and ent.abs().max() <= 1e-5
        assert ((logz - (c["x"].float() @ c["wv"].float().t() + c["bv"])[:, 0]).abs() <= 1e-5 * (1 + logz.abs())).all()
        for t in fl.fb_affine_logprobs_grad(c["x"], c["wv"], c["tokens"], logz, ent, c["g"], c["h"], c["bv"]):
            # (p = 1 to some 1e-6: the gradient of a certainty)
            assert t.abs().max() <= 1e-5 * M * 20


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("K", [3, 40])
def test_no_rows_of_any_type(fl, dtype, K):
    """Sums over no rows are zeros, whatever the workspace held: products that leave at once (K = 40) and by way of memory (3)."""
    import torch
    c = make(0, 66, K, dtype, 1)
    out = run(fl, c)
    for t in out:
        assert t is not None and not t.any() and not torch.isnan(t).any()
    none = torch.empty(0, device="cuda")
    for t in fl.fb_affine_logprobs_grad(c["x"], c["wv"], c["tokens"], none, none, none, None, c["bv"]):
        assert not t.any() and not torch.isnan(t).any()
