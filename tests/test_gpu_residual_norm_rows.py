"""The residual norm over many rows of widths that are not whole 16-byte pieces: workgroups that take row after row, so that rows are asked
for ahead, sums of columns run over several rows, and outputs in place of inputs are written while the next rows come.  Checks and
bounds are those of test_gpu_residual_norm.py."""
from __future__ import annotations

import pytest

from test_gpu_residual_norm import KINDS, check_forward, check_grad, fl, make, rows  # noqa: F401  (fl: the fixture)

pytestmark = pytest.mark.gpu


# forward, up to 2048 workgroups of 4, 2 or 1 rows (1024 of rows above 2048); backward up to 512
@pytest.mark.parametrize("R,H", [(9000, 77), (9000, 7), (5000, 777), (2500, 1357), (2500, 2357), (2500, 4095), (2500, 5094)])
@pytest.mark.parametrize("dtype,gap,wdtype", [("bfloat16", 0, "float32"), ("float16", 3, "float16"), ("bfloat16", 5, "bfloat16")])
def test_forward(fl, R, H, dtype, gap, wdtype):  # noqa: F811
    k = R + H + gap
    for v in range(2):
        check_forward(fl, R, H, dtype, gap, *KINDS[(k + 2 * v) % 7], wdtype, seed=k + v)


@pytest.mark.parametrize("R,H", [(5000, 77), (5000, 7), (2600, 777), (1300, 1357), (1300, 2357), (1300, 4095), (1300, 5094), (1300, 8191), (1300, 6144)])
@pytest.mark.parametrize("dtype,gap,wdtype", [("bfloat16", 0, "float32"), ("float16", 3, "float16"), ("bfloat16", 5, "bfloat16"), ("float32", 0, "float32")])
def test_gradient(fl, R, H, dtype, gap, wdtype):  # noqa: F811
    k = R + H + gap
    for v in range(2):
        inner, outer, gate, _ = KINDS[(k + 2 * v) % 7]
        check_grad(fl, R, H, dtype, gap, inner, outer, gate, wdtype, seed=k + v, with_ds=v != 1)


FORMS = {"none": 0, "layer": 1, "rms": 2}


@pytest.mark.parametrize("R,H", [(9000, 41), (5000, 1001), (2500, 3003), (2500, 5005)])
@pytest.mark.parametrize("inner,outer", [("rms", "layer"), ("none", "none"), ("none", "rms"), ("layer", "none")])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
def test_outputs_in_place_of_inputs(fl, R, H, inner, outer, dtype):  # noqa: F811
    """Through the C calls, each output of rows on each input of rows in turn: the bits of outputs of their own."""
    import torch

    import paper_2112_00709_amd as base
    code, ld = {"float32": 0, "bfloat16": 1, "float16": 2}[dtype], H + 3
    h, r, g, _ = make(R, H, dtype, 3, "none", "none", "rows", True, "float32")
    ds, dy = rows(R, H, dtype, 3, 8), rows(R, H, dtype, 3, 9)
    s, y, stats = fl.fb_residual_norm(h, r, g, scale=0.7, inner=inner, outer=outer, want_stats=True)
    st = torch.cuda.current_stream().cuda_stream

    def apart(*ts):
        """Copies of the rows in memory of their own, at the same distance."""
        out = []
        for t in ts:
            wide = torch.full((R, ld), 7.0, device="cuda").to(t.dtype)
            wide[:, :H] = t
            out.append(wide)
        return out

    for turn in range(3):
        a = apart(h, r, g)
        to_s, to_y = a[turn], a[(turn + 1) % 3]
        base._check(fl.lib().fb_residual_norm(a[0].data_ptr(), ld, a[1].data_ptr(), ld, a[2].data_ptr(), ld, 0.7, FORMS[inner], None, None, FORMS[outer], None, None, 0,
                                              R, H, code, 1e-5, to_s.data_ptr(), ld, to_y.data_ptr() if outer != "none" else None, ld, None, st))
        assert torch.equal(to_s[:, :H], s)
        if outer != "none":
            assert torch.equal(to_y[:, :H], y)
        assert all((t[:, H:] == 7.0).all() for t in a)

    want = fl.fb_residual_norm_grad(ds, dy if outer != "none" else None, h, s, stats, g, scale=0.7, inner=inner, outer=outer, want_dinner=False, want_douter=False)
    for turn in range(5):
        a = apart(ds, dy, h, s, g)                          # (dy and s are read with an outer norm alone)
        outs = [a[(turn + k) % 5] for k in (0, 2, 4)]
        base._check(fl.lib().fb_residual_norm_grad(a[0].data_ptr(), ld, a[1].data_ptr(), ld, a[2].data_ptr(), ld, a[3].data_ptr(), ld, stats.data_ptr(), a[4].data_ptr(), ld, 0.7,
                                                   FORMS[inner], None, None, FORMS[outer], None, 0, R, H, code, outs[0].data_ptr(), ld, outs[1].data_ptr(), ld,
                                                   outs[2].data_ptr(), ld, None, None, None, None, None, 0, st))
        for out, t in zip(outs, want):
            assert torch.equal(out[:, :H], t)
        assert all((t[:, H:] == 7.0).all() for t in a)
