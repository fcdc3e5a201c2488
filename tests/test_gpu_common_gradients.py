"""Gradients of log probabilities whose g is one number in all rows (a mean loss) or whose rows that count are few, in 16 bits: the rounding of g is
not in every gradient.

Logits are nearly equal, V = 4096: p is 2^-12 up to some r, so dz is g (1 - p) at a row's token and -g p elsewhere.  dz is rounded to 16
bits times a factor that makes |g| a power of two: the token's entry is then off by p of its size (1 - p rounds to 1) and the others by r (they
round to 2^-12).  Everything else is in single precision: sums of n terms are off by at most 2 (n / 16 + 40) u of their sizes, p by
the logits' and log Z's 64 u.  The outputs are rounded once, half a step.  g is half a step off a number of the type: rounded as it is, that
alone would be another half step in every element of dx and dweight."""
from __future__ import annotations

import pytest

from test_gpu_vocabulary import fl  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
V, K = 4096, 16


@pytest.mark.parametrize("M", [300, 2000, 3000])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("live", [1, 2, None])
@pytest.mark.parametrize("size", [1.0, 2.0 ** -9, 48.0])
def test_one_gradient_in_all_rows(fl, M, dtype, live, size):  # noqa: F811
    import torch
    t = getattr(torch, dtype)
    half = torch.finfo(t).eps / 2
    gen = torch.Generator().manual_seed(M)
    x = (torch.randn((M, K), generator=gen) * 2.0 ** -13).cuda().to(t)
    w = (torch.randn((V, K), generator=gen) * 2.0 ** -5).cuda().to(t)
    tokens = torch.randperm(V, generator=gen)[:M].to(torch.int32).cuda()
    if live is not None:
        tokens[torch.randperm(M, generator=gen)[live:].cuda()] = -1
    g = torch.full((M,), -size * (1 + half), device="cuda")
    counts = (tokens >= 0)[:, None]
    _, ent, logz = fl.fb_affine_logprobs(x, w, tokens)
    dx, dw, db = fl.fb_affine_logprobs_grad(x, w, tokens, logz, ent, g)
    xd, wd, gd = x.double().masked_fill(~counts, 0), w.double(), g.double()[:, None]
    z = xd @ wd.t().contiguous()
    p = torch.exp(z - z.logsumexp(1, keepdim=True))
    far = (p * V - 1).abs()
    assert float(far.max()) < half / 2                       # (so that p rounds to 2^-12, below which a half step is half as wide)
    at = tokens.clamp_min(0).long()[:, None]
    dz, off = -gd * p, gd.abs() * p * (far + 64 * U)
    dz.scatter_add_(1, at, gd)
    off.scatter_(1, at, gd.abs() * p.gather(1, at) * (1 + 64 * U))
    dz, off = dz.masked_fill(~counts, 0), off.masked_fill(~counts, 0)

    def check(got, want, tol, half):
        tol = tol + half * (want.abs() + tol) + (2.0 ** -25 if got.dtype == torch.float16 else 0.0)
        bad = ~((got.double() - want).abs() <= 1.001 * tol)
        assert not bad.any(), (int(bad.sum()), got[bad][:4], want[bad][:4])

    check(dx, dz @ wd, off @ wd.abs() + 2 * (V / 16 + 40) * U * (dz.abs() @ wd.abs()), half)
    check(dw, dz.t().contiguous() @ xd, off.t().contiguous() @ xd.abs() + 2 * (M / 16 + 40) * U * (dz.abs().t().contiguous() @ xd.abs()), half)
    # (summed before the rounding: what it is off by is not in dbias)
    check(db, dz.sum(0), (gd.abs() * p * 64 * U).masked_fill(~counts, 0).sum(0) + (M / 16 + 40) * U * dz.abs().sum(0), 2 * U)
