"""Logits of long rows in 16 bits: terms far below the running sum are not lost one by one, where tiles are of up to 128.

Rows are made for it: the first product is 4, the others 2^-28 each.  A matrix instruction adds 16 of them, 2^-24, which is a quarter of
half a step of 4: in one chain over k nothing of them would be left, K 2^-28 = 2^-13 in all.  In shares of 512 k a running sum has
32 instructions, each off by at most 2 u of 4 (it may truncate), and K / 512 shares are added with one rounding each: off by at most
4 (64 + K / 512 + 4) u, a quarter of 2^-13 for K = 32768."""
from __future__ import annotations

import pytest

from test_gpu_vocabulary import fl  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
K = 32768
OFF = 4 * (64 + K / 512 + 4) * U


def made(M, V, dtype):
    """x, weight: all logits are 4 + (K - 1) 2^-28."""
    import torch
    t = getattr(torch, dtype)
    x, w = (torch.full((n, K), 2.0 ** -14, device="cuda") for n in (M, V))
    x[:, 0] = w[:, 0] = 2.0
    return x.to(t), w.to(t), 4 + (K - 1) * 2.0 ** -28


@pytest.mark.parametrize("M,V", [(65, 1), (70, 40), (300, 130)])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_forward(fl, M, V, dtype):  # noqa: F811
    import math

    import torch
    x, w, z = made(M, V, dtype)
    _, _, logz = fl.fb_affine_logprobs(x, w, torch.zeros(M, dtype=torch.int32, device="cuda"))
    # (log Z: the logit, and log V from a sum of ones with up to V / 64 + 8 roundings and a library's logarithm)
    assert ((logz.double() - z - math.log(V)).abs() <= OFF + (V / 64 + 16) * U + 2 * U * abs(z + math.log(V))).all()


@pytest.mark.parametrize("M,V", [(1, 1), (17, 40), (70, 40), (300, 130)])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_gradient(fl, M, V, dtype):  # noqa: F811
    """With the log Z that is right: of tokens beyond the vocabulary dbias is sum p, M / V."""
    import math

    import torch
    x, w, z = made(M, V, dtype)
    logz = torch.full((M,), z + math.log(V), device="cuda")
    tokens = torch.full((M,), V, dtype=torch.int32, device="cuda")
    _, _, db = fl.fb_affine_logprobs_grad(x, w, tokens, logz, None, torch.full((M,), -1.0, device="cuda"))
    # (p: the logit, log Z's rounding and the exponential's 16 u; M of them added with at most M / 16 + 8 roundings)
    off = OFF + U * abs(z + math.log(V)) + 16 * U + (M / 16 + 8) * U
    assert ((db.double() * V / M - 1).abs() <= off * 1.01).all()
