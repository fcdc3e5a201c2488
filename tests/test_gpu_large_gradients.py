"""Gradients of many rows against the definitions in 64 bits, by the ways of dx that only large calls take: whole rounds of large tiles and
then the rest of the rows by smaller ones; pieces of the vocabulary that add up in single precision where each piece's product leaves at
once, with and without that cut.  (test_gradient_plans_host.py holds that these sizes go these ways.)  Bounds are those of the files
that the checks come from."""
from __future__ import annotations

import pytest

import test_gpu_affine as affine
import test_gpu_gated as gated
import test_gpu_vocabulary as vocabulary
from test_gpu_vocabulary import fl  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,V,K,dtype", [(69120, 300, 1024, "bfloat16"), (69120, 300, 1024, "float16"), (40000, 7000, 1024, "bfloat16"), (40000, 7000, 1024, "float16"),
                                         (70000, 4200, 256, "bfloat16"), (70000, 4200, 256, "float16"), (70000, 4200, 256, "float32")])
def test_log_probabilities(fl, M, V, K, dtype):  # noqa: F811
    """Rows that do not count, with NaN in x, on both sides of every cut; tokens at the ends of the pieces."""
    import torch
    x, w, b, tokens = vocabulary.inputs(M, V, K, dtype, 0, M + V)
    for i in (32768, 65536):
        if i < M:
            tokens[[i - 2, i + 1, i + 2]] = torch.tensor([-1, -1, -7], dtype=torch.int32, device="cuda")
            x[[i - 2, i + 1, i + 2]] = float("nan")
            tokens[[i - 1, i]] = torch.tensor([V - 1, 0], dtype=torch.int32, device="cuda")
            x[[i - 1, i]] = 0.25
    x[tokens < 0] = float("nan")
    b[[0, V - 1]] = 0.5
    got = vocabulary.check_grad(fl, x, w, b, tokens, vocabulary.numbers(M, 5), vocabulary.numbers(M, 6, 0.1))
    assert not torch.isnan(got[1]).any()


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("activation,dy_type", [("none", "same"), ("gelu", "f32")])
def test_affine_layer(fl, dtype, activation, dy_type):  # noqa: F811
    affine.check_grad(fl, 69120, 300, 1024, dtype, 0, activation, dy_type)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_gated_layer(fl, dtype):  # noqa: F811
    gated.check_grad(fl, 69120, 150, 1024, dtype, 0, "silu")
