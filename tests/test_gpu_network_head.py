"""The last layers together: as differentiable functions against PyTorch's own gradients in 64 bits, and the example that
trains them with the LF-MMI objective and serves single frames."""
from __future__ import annotations

import os
import sys

import pytest

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module")
def fa():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_2112_00709_amd as base
    from paper_2112_00709_amd import autograd
    base.POISON_NEW_BUFFERS = True
    return autograd


def reference(p, hidden, tokens, ce, ent_w, g_emis):
    """The head in 64 bits with PyTorch's functions: emissions, and the gradients of a loss that is linear in them plus the
    frame terms."""
    import torch
    import torch.nn.functional as F
    q = {k: v.detach().double().cpu().requires_grad_(True) for k, v in p.items()}
    h = hidden.detach().double().cpu().requires_grad_(True)
    n = h.shape[-1]
    x = F.layer_norm(h, (n,), q["norm0_w"], q["norm0_b"])
    x = F.gelu(x @ q["hidden_w"].t() + q["hidden_b"])
    x = x @ q["back_w"].t() + q["back_b"] + h
    x = F.layer_norm(x, (n,), q["norm1_w"], q["norm1_b"])
    emis = x @ q["out_w"].t() + q["out_b"]
    logp = torch.log_softmax(emis, -1)
    t = tokens.long().cpu()
    live = (t >= 0).double()
    lp = logp.gather(-1, t.clamp_min(0)[..., None])[..., 0] * live
    ent = -(logp.exp() * logp).sum(-1) * live
    loss = (emis * g_emis.double().cpu()).sum() + ce * lp.sum() + ent_w * ent.sum()
    loss.backward()
    return emis.detach(), {k: v.grad for k, v in q.items()}, h.grad


# In single precision every operator is good to some 1e-6 of its output's size and there are a dozen of them behind one another:
# 1e-4 in the 2-norm.  In 16 bits each of a dozen roundings (activations, weights, gradients) adds h / sqrt 3 of its size in the
# 2-norm, for weights and activations alike: sqrt(24) h / sqrt 3 = 3 h; 6 h is held (2^-8, 2^-11).
@pytest.mark.parametrize("dtype,tol", [("float32", 1e-4), ("bfloat16", 6 * 2.0 ** -8), ("float16", 6 * 2.0 ** -11)])
def test_gradients_of_the_whole_head(fa, dtype, tol):
    import torch

    from network_head import Head
    t = getattr(torch, dtype)
    gen = torch.Generator().manual_seed(4)
    hidden = torch.randn((3, 37, 72), generator=gen).cuda().to(t).requires_grad_(True)
    head = Head(72, 104, 50, t, seed=3)
    tokens = torch.randint(0, 50, (3, 37), generator=gen, dtype=torch.int32).cuda()
    tokens[1, 20:] = -1
    g_emis = torch.randn((3, 37, 50), generator=gen).cuda()
    emis = head(hidden)
    lp, ent, logz, ids, best = fa.token_logprobs(emis, tokens, top=3)
    assert not logz.requires_grad and not best.requires_grad
    ((emis * g_emis).sum() + 0.7 * lp.sum() + 0.2 * ent.sum()).backward()
    want_emis, want, want_h = reference(head.params, hidden, tokens, 0.7, 0.2, g_emis)

    def far(a, b):
        return float((a.detach().double().cpu() - b).norm() / b.norm())

    assert far(emis, want_emis) <= tol
    for k, v in head.params.items():
        assert v.grad.dtype == torch.float32 and far(v.grad, want[k]) <= tol, k
    assert hidden.grad.dtype == t and far(hidden.grad, want_h) <= tol


def test_parts_that_need_no_gradient(fa):
    import torch
    x = torch.randn((5, 16), device="cuda", requires_grad=True)
    w = torch.randn((8, 16), device="cuda")
    y = fa.affine(x, w, activation="silu", residual=torch.zeros((5, 8), device="cuda"))
    y.sum().backward()                                     # (a gradient that is one number, expanded)
    z = x.detach().double() @ w.double().t()
    s = torch.sigmoid(z)
    assert torch.allclose(x.grad.double(), (s + z * s * (1 - s)) @ w.double(), rtol=1e-4, atol=1e-5)
    n = fa.layer_norm(x.detach(), torch.ones(16, device="cuda", requires_grad=True))
    assert n.requires_grad
    r = torch.randn((5, 8), device="cuda", requires_grad=True)
    fa.affine(x.detach(), w, residual=r).sum().backward()
    assert torch.equal(r.grad, torch.ones_like(r))
    logits = torch.randn((4, 9), device="cuda", requires_grad=True)
    lp = fa.token_logprobs(logits, torch.arange(4, dtype=torch.int32, device="cuda"))[0]
    lp.sum().backward()
    want = torch.zeros(4, 9)
    want[range(4), range(4)] = 1
    assert torch.allclose(logits.grad.cpu(), want - torch.softmax(logits.detach().cpu(), 1), atol=1e-6)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_the_example_learns_and_serves(fa, dtype):
    import torch

    import network_head as nh
    w, den, num, hidden = nh.setup(K=600, B=5, D=60, H=96, dtype=dtype)
    head = nh.Head(96, 128, w.D, getattr(torch, dtype))
    log = nh.train(head, hidden, w, den, num, 8)
    print("objective per step:", [round(l[0], 4) for l in log], flush=True)
    assert all(l == l and abs(l) < 1e6 for step in log for l in step)
    assert log[-1][0] > log[0][0] and log[-1][1] > log[0][1]
    ids, best, ents = nh.serve(head, hidden[0, :3], top=4)
    with torch.no_grad():
        logp = torch.log_softmax(head(hidden[0, :3]).double().cpu(), -1)
    # a frame alone runs in another kernel than a batch: the same sums in another order
    assert ids.shape == (3, 4) and torch.allclose(best.double().cpu(), logp.gather(1, ids.long().cpu()), rtol=0, atol=1e-2 if dtype == "bfloat16" else 1e-4)
    assert ((best[:, :-1] >= best[:, 1:]).all()) and (ents > 0).all()
    den.destroy()
    num.destroy()
