"""A feed-forward block and a token loss as they are used together: residual norm, gated layer, the way back down, residual norm, log
probabilities from hidden frames, as differentiable functions against PyTorch's own gradients in 64 bits."""
from __future__ import annotations

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fa():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_2112_00709_amd as base
    from paper_2112_00709_amd import autograd
    base.POISON_NEW_BUFFERS = True
    return autograd


def parameters(H, F, V, seed=0):
    import torch
    gen = torch.Generator().manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen) * shape[-1] ** -0.5

    p = dict(in_w=1 + 0.2 * torch.randn(H, generator=gen), norm0_w=1 + 0.2 * torch.randn(H, generator=gen), norm0_b=0.1 * torch.randn(H, generator=gen),
             gate=0.5 + 0.2 * torch.randn(H, generator=gen), up_w=normal(2 * F, H), up_b=0.1 * torch.randn(2 * F, generator=gen), down_w=normal(H, F),
             norm1_w=1 + 0.2 * torch.randn(H, generator=gen), out_w=normal(V, H) * 2, out_b=torch.randn(V, generator=gen))
    return {k: v.cuda().requires_grad_(True) for k, v in p.items()}


def block(fa, p, t, h, tokens):
    """-> (sum that goes on, log probabilities, entropy)."""
    s, y = fa.residual_norm(h, None, None, 1.0, "rms", p["in_w"], None, "layer", p["norm0_w"], p["norm0_b"])
    u = fa.gated_affine(y, p["up_w"].to(t), p["up_b"])
    u = fa.affine(u, p["down_w"].to(t))
    s, y = fa.residual_norm(u, s, p["gate"], 0.5, "none", outer="rms", weight=p["norm1_w"])
    return s, *fa.affine_logprobs(y, p["out_w"].to(t), tokens, p["out_b"])


def reference(p, h, tokens, g_s, ce, ent_w):
    import torch
    import torch.nn.functional as F
    q = {k: v.detach().double().cpu().requires_grad_(True) for k, v in p.items()}
    x = h.detach().double().cpu().requires_grad_(True)
    n = (x.shape[-1],)
    s = F.rms_norm(x, n, q["in_w"], 1e-5)
    y = F.layer_norm(s, n, q["norm0_w"], q["norm0_b"])
    a, b = (y @ q["up_w"].t() + q["up_b"]).chunk(2, -1)
    s = s + 0.5 * q["gate"] * ((F.silu(a) * b) @ q["down_w"].t())
    y = F.rms_norm(s, n, q["norm1_w"], 1e-5)
    logp = torch.log_softmax(y @ q["out_w"].t() + q["out_b"], -1)
    t = tokens.long().cpu()
    live = (t >= 0).double()
    lp = logp.gather(-1, t.clamp_min(0)[..., None])[..., 0] * live
    ent = -(logp.exp() * logp).sum(-1) * live
    ((s * g_s.double().cpu()).sum() + ce * lp.sum() + ent_w * ent.sum()).backward()
    return s.detach(), lp.detach(), ent.detach(), {k: v.grad for k, v in q.items()}, x.grad


# Tolerances in the 2-norm, as for the other layers' run: in single precision some 1e-6 of an operator's size for each of a dozen, 1e-4;
# in 16 bits a dozen roundings each way of h / sqrt 3 of their size, 3 h, of which 6 h are held.
TYPES = [("float32", 1e-4), ("bfloat16", 6 * 2.0 ** -8), ("float16", 6 * 2.0 ** -11)]


@pytest.mark.parametrize("dtype,tol", TYPES)
@pytest.mark.parametrize("B,N,H,F,V", [(3, 37, 72, 104, 50), (2, 9, 33, 17, 301), (7, 61, 264, 520, 2050)])
def test_gradients_of_the_whole_run(fa, dtype, tol, B, N, H, F, V):
    import torch
    t = getattr(torch, dtype)
    gen = torch.Generator().manual_seed(4)
    h = torch.randn((B, N, H), generator=gen).cuda().to(t).requires_grad_(True)
    p = parameters(H, F, V)
    tokens = torch.randint(0, V, (B, N), generator=gen, dtype=torch.int32).cuda()
    tokens[1, N // 2:] = -1
    g_s = torch.randn((B, N, H), generator=gen).cuda()
    s, lp, ent, logz = block(fa, p, t, h, tokens)
    assert not logz.requires_grad and s.dtype == t and lp.dtype == torch.float32
    ((s * g_s).sum() + 0.7 * lp.sum() + 0.2 * ent.sum()).backward()
    want_s, want_lp, want_ent, want, want_h = reference(p, h, tokens, g_s, 0.7, 0.2)

    def far(a, b):
        return float((a.detach().double().cpu() - b).norm() / b.norm())

    assert far(s, want_s) <= tol and far(lp, want_lp) <= tol and far(ent, want_ent) <= tol
    for k, v in p.items():
        assert v.grad.dtype == torch.float32 and far(v.grad, want[k]) <= tol, (k, far(v.grad, want[k]))
    assert h.grad.dtype == t and far(h.grad, want_h) <= tol


def test_one_step_is_the_same_alone_as_among_others(fa):
    """Single frames, as a recogniser that is fed frame by frame asks for them: other kernels, the same to the sums' order."""
    import torch
    t = torch.float32
    p = parameters(264, 520, 2050)
    h = torch.randn((100, 264), generator=torch.Generator().manual_seed(3)).cuda()
    tokens = torch.arange(100, dtype=torch.int32, device="cuda")
    with torch.no_grad():
        many = block(fa, p, t, h, tokens)
        for i in (0, 57, 99):
            for a, b in zip(block(fa, p, t, h[i:i + 1], tokens[i:i + 1]), many):
                # (some 1e-6 of the sizes, 10 at most, through three layers)
                assert ((a[0] - b[i]).abs() <= 1e-4).all()


def test_parts_that_need_no_gradient(fa):
    import torch
    x = torch.randn((5, 16), device="cuda", requires_grad=True)
    w = torch.randn((8, 16), device="cuda")
    tokens = torch.arange(5, dtype=torch.int32, device="cuda")
    y = fa.gated_affine(x, w)
    y.sum().backward()                                     # (a gradient that is one number, expanded)
    z = x.detach().double().requires_grad_(True)
    a, b = (z @ w.double().t()).chunk(2, 1)
    (torch.nn.functional.silu(a) * b).sum().backward()
    assert torch.allclose(x.grad.double(), z.grad, rtol=1e-4, atol=1e-5)
    x.grad = None
    lp, ent, _ = fa.affine_logprobs(x, w, tokens)
    ent.sum().backward()                                   # (one of both alone)
    z = x.detach().double().requires_grad_(True)
    logp = torch.log_softmax(z @ w.double().t(), 1)
    (-(logp.exp() * logp).sum()).backward()
    assert torch.allclose(x.grad.double(), z.grad, rtol=1e-4, atol=1e-5)
    wg = w.clone().requires_grad_(True)
    fa.affine_logprobs(x.detach(), wg, tokens)[0].sum().backward()
    assert wg.grad.shape == w.shape
    r = torch.randn((5, 16), device="cuda", requires_grad=True)
    s, y = fa.residual_norm(x.detach(), r, scale=2.0, outer="none")
    assert y is None
    s.sum().backward()
    assert torch.equal(r.grad, torch.ones_like(r))
    for use in (0, 1):                                     # (the sum or the norm alone)
        h, r = (torch.randn((5, 16), device="cuda", requires_grad=True) for _ in range(2))
        gate = torch.randn((5, 16), device="cuda", requires_grad=True)
        c = torch.randn((5, 16), device="cuda")
        (fa.residual_norm(h, r, gate, 0.3)[use] * c).sum().backward()
        q = [t.detach().double().requires_grad_(True) for t in (h, r, gate)]
        s = q[1] + 0.3 * q[2] * q[0]
        ((s if use == 0 else torch.nn.functional.layer_norm(s, (16,))) * c).sum().backward()
        for t, want in zip((h, r, gate), q):
            assert torch.allclose(t.grad.double(), want.grad, rtol=1e-4, atol=1e-5)


def test_the_same_tensor_twice(fa):
    """h as its own residual, and one gate for both: gradients add up."""
    import torch
    x = torch.randn((6, 40), device="cuda", requires_grad=True)
    s, y = fa.residual_norm(x, x, x, 0.5, "layer")
    (s * 0.1 + y * y * y).sum().backward()
    z = x.detach().double().requires_grad_(True)
    f = torch.nn.functional.layer_norm
    s = z + 0.5 * z * f(z, (40,))
    y = f(s, (40,))
    (s * 0.1 + y * y * y).sum().backward()
    assert torch.allclose(x.grad.double(), z.grad, rtol=1e-3, atol=1e-4)


@pytest.mark.parametrize("which", ["logprobs", "entropy", "logz", "all"])
def test_results_may_be_changed_in_place(fa, which):
    import torch
    gen = torch.Generator().manual_seed(5)
    x0, w = torch.randn((6, 24), generator=gen).cuda(), torch.randn((70, 24), generator=gen).cuda()
    tokens = torch.randint(0, 70, (6,), generator=gen, dtype=torch.int32).cuda()
    pad = torch.tensor([False, True, False, False, True, False], device="cuda")

    def grad(inplace):
        x = x0.clone().requires_grad_(True)
        lp, ent, logz = fa.affine_logprobs(x, w, tokens)
        if inplace:
            if which in ("logprobs", "all"):
                lp.masked_fill_(pad, 0.0).mul_(0.5)
            if which in ("entropy", "all"):
                ent.masked_fill_(pad, 0.0).mul_(0.25)
            if which in ("logz", "all"):
                logz.add_(1.0)
        else:
            if which in ("logprobs", "all"):
                lp = lp.masked_fill(pad, 0.0) * 0.5
            if which in ("entropy", "all"):
                ent = ent.masked_fill(pad, 0.0) * 0.25
        (lp.sum() + 0.3 * ent.sum()).backward()
        return x.grad

    assert torch.equal(grad(True), grad(False))


def test_a_training_step_replayed(fa):
    """Forward and backward pass recorded into a graph, replayed with new frames: the bits of the eager step."""
    import torch
    t = torch.bfloat16
    p = parameters(136, 200, 300)
    leaves = list(p.values())
    h = torch.randn((70, 136), device="cuda").to(t).requires_grad_(True)
    tokens = torch.randint(-1, 300, (70,), dtype=torch.int32, device="cuda")

    def step():
        s, lp, ent, _ = block(fa, p, t, h, tokens)
        out = torch.autograd.grad((s.float() * 0.1).mean() + lp.mean() + 0.1 * ent.mean(), [h, *leaves])
        return [x.clone() for x in (s.detach(), lp.detach(), ent.detach(), *out)]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for seed in (1, 2, 3):
        with torch.no_grad():
            h.copy_(torch.randn((70, 136), generator=torch.Generator().manual_seed(seed)).cuda())
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, step()):
            assert torch.equal(a, b)
