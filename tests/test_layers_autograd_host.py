"""What the differentiable last layers ask of the operators, without a GPU: nothing is formed for a backward pass that cannot
follow."""
import pytest
import torch

from paper_2112_00709_amd import autograd as fa
from paper_2112_00709_amd import layers as fl


@pytest.fixture
def asked(monkeypatch):
    """The operators replaced by ones that note what they are asked for beyond their result."""
    seen = []

    def affine(x, weight, bias=None, activation="none", residual=None, out_dtype=None, want_preact=False):
        seen.append(want_preact)
        y = x @ weight.t()
        return (y, y.clone()) if want_preact else y

    def layer_norm(x, weight=None, bias=None, eps=1e-5, want_stats=False):
        seen.append(want_stats)
        y = x.clone()
        return (y, x.mean(-1), x.mean(-1)) if want_stats else y

    monkeypatch.setattr(fl, "fb_affine", affine)
    monkeypatch.setattr(fl, "fb_layer_norm", layer_norm)
    return seen


CALLS = [lambda x, w, b: fa.affine(x, w, activation="relu"), lambda x, w, b: fa.layer_norm(x, b)]


@pytest.mark.parametrize("call", CALLS)
def test_nothing_is_kept_where_no_gradient_can_be_asked_for(asked, call):
    x, w, b = torch.randn(3, 4), torch.randn(4, 4, requires_grad=True), torch.randn(4, requires_grad=True)
    with torch.no_grad():
        assert not call(x, w, b).requires_grad
    with torch.inference_mode():
        call(x, w, b)
    assert not call(x, w.detach(), b.detach()).requires_grad
    assert asked == [False, False, False]


@pytest.mark.parametrize("call", CALLS)
def test_what_a_backward_pass_takes_is_kept_where_one_can_follow(asked, call):
    x, w, b = torch.randn(3, 4), torch.randn(4, 4, requires_grad=True), torch.randn(4, requires_grad=True)
    assert call(x, w, b).requires_grad
    assert call(x.clone().requires_grad_(True), w.detach(), b.detach()).requires_grad
    with torch.no_grad():
        with torch.enable_grad():
            call(x, w, b)
    assert asked == [True, True, True]
