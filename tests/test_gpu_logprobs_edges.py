"""Gradient of token log probabilities at the ends of the numbers: ruled-out alternatives under large incoming gradients."""
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


@pytest.mark.parametrize("V", [5, 130, 1500, 9001])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("h", [1e9, 1e20, -1e30])
def test_ruled_out_alternatives_under_a_large_gradient_of_the_entropy(fl, V, dtype, h):
    """p log p is 0 where p is, whatever it is multiplied by (scaled losses).  Tolerance: that of the gradient's own test, 60 u of
    h (2 + 2 log V), and the result's rounding."""
    import torch
    gen = torch.Generator().manual_seed(V)
    x = torch.randn((4, V), generator=gen)
    x[:, ::2] = -math.inf
    x[1, 1:] = torch.finfo(torch.float32).min / 2
    x[2] = -math.inf
    x[2, V - 1] = 3.0
    x = x.to(getattr(torch, dtype)).cuda()
    x[0, 1] = 0.5
    tokens = torch.tensor([1, 0, V - 1, 1], dtype=torch.int32, device="cuda")
    _, ent, z, _, _ = fl.fb_token_logprobs(x, tokens)
    g, hh = torch.zeros(4, device="cuda"), torch.full((4,), h, device="cuda")
    got = fl.fb_token_logprobs_grad(x, tokens, z, ent, g, hh).double().cpu()
    xd, zd, ed = x.double().cpu(), z.double().cpu(), ent.double().cpu()
    lp = xd - zd[:, None]
    p = lp.exp()
    want = -hh.double().cpu()[:, None] * torch.where(p > 0, p * (torch.where(p > 0, lp, 0.0) + ed[:, None]), 0.0)
    assert torch.isfinite(got).all()
    tol = 60 * 2.0 ** -24 * abs(h) * (2 + 2 * math.log(V + 1)) + (2.0 ** -8 if dtype == "bfloat16" else 2.0 ** -24) * want.abs()
    assert ((got - want).abs() <= tol).all()
    assert (got[p == 0] == 0).all()
