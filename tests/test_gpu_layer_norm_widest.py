"""Layer norm's gradient at the widest rows that the header allows."""
from __future__ import annotations

import pytest

pytestmark = pytest.mark.gpu


def test_the_widest_row():
    """One row: dbias is dy itself, dweight dy times what the statistics make of x (three roundings: 4 u)."""
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_2112_00709_amd as base
    from paper_2112_00709_amd import layers as fl
    fl.lib()
    base.POISON_NEW_BUFFERS = True
    H = (1 << 28) - 1
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, dy = (torch.randn((1, H), generator=gen, device="cuda") for _ in range(2))
    mean, rstd = torch.full((1,), 0.25, device="cuda"), torch.full((1,), 1.5, device="cuda")
    _, dw, db = fl.fb_layer_norm_grad(dy, x, mean, rstd, want_dx=False)
    assert torch.equal(db, dy[0])
    want = dy[0] * ((x[0] - 0.25) * 1.5)
    assert ((dw - want).abs() <= 4 * 2.0 ** -24 * want.abs()).all()
