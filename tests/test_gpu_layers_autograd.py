"""The last layers' differentiable functions as training loops use them: results changed in place, and calls after which no
gradient can be asked for."""
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


@pytest.mark.parametrize("which", ["none", "logprobs", "entropy", "logz", "all"])
@pytest.mark.parametrize("V", [7, 3000])
def test_results_may_be_changed_in_place(fa, which, V):
    """Masking or scaling a result in place is part of the differentiated program; the same gradient as with a new tensor."""
    import torch
    gen = torch.Generator().manual_seed(V)
    logits = torch.randn((6, V), generator=gen).cuda()
    tokens = torch.randint(0, V, (6,), generator=gen, dtype=torch.int32).cuda()
    pad = torch.tensor([False, True, False, False, True, False], device="cuda")

    def grad(inplace):
        x = logits.clone().requires_grad_(True)
        lp, ent, logz, _, _ = fa.token_logprobs(x, tokens, top=3)
        if inplace:
            if which in ("logprobs", "all"):
                lp.masked_fill_(pad, 0.0).mul_(0.5)
            if which in ("entropy", "all"):
                ent.masked_fill_(pad, 0.0).mul_(0.25)
            if which in ("logz", "all"):
                logz.add_(1.0)
                with torch.no_grad():
                    logz.zero_()
        else:
            if which in ("logprobs", "all"):
                lp = lp.masked_fill(pad, 0.0) * 0.5
            if which in ("entropy", "all"):
                ent = ent.masked_fill(pad, 0.0) * 0.25
        (lp.sum() + 0.3 * ent.sum()).backward()
        return x.grad

    assert torch.equal(grad(True), grad(False))


def test_results_of_the_plain_calls_are_tensors_of_their_own(fa):
    import torch

    from paper_2112_00709_amd import layers as fl
    x = torch.randn((5, 40), device="cuda")
    scale = torch.ones(5, device="cuda", requires_grad=True)
    lp, ent, logz, _, _ = fl.fb_token_logprobs(x, torch.zeros(5, dtype=torch.int32, device="cuda"))
    _, mean, rstd = fl.fb_layer_norm(x, want_stats=True)
    for t in (lp, ent, logz, mean, rstd):
        before = t._version
        t.mul_(scale)                                      # (refused of one of several views)
        assert t.requires_grad and t._version == before + 1


def test_other_streams_and_leading_shapes_give_the_same_bits(fa):
    import torch

    from paper_2112_00709_amd import layers as fl
    gen = torch.Generator().manual_seed(1)
    for R, V, top in ((12, 9000, 3), (12, 84, 30), (4, 70001, 5), (2400, 700, 4)):
        x = (3 * torch.randn((R, V), generator=gen)).bfloat16().cuda()
        tokens = torch.randint(-1, V, (R,), generator=gen, dtype=torch.int32).cuda()
        x[tokens < 0] = float("nan")
        x[2] = -float("inf")
        flat = fl.fb_token_logprobs(x, tokens, top=top)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            other = fl.fb_token_logprobs(x.view(2, R // 2, V), tokens.view(2, R // 2), top=top)
        s.synchronize()
        for a, b in zip(flat, other):
            assert not torch.isnan(a).any() and torch.equal(a, b.view(a.shape))
