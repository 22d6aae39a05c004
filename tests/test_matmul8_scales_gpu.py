"""8-bit products whose scales are far from one while their products are not: whatever form runs, a block's sum meets the product of its two
scales and nothing else that could leave fp32's range.  (A block's sum reaches 2^24, so times 2^110 alone it would be infinite; times 2^-125
alone a small one would lose bits.)

Tolerance as for any scales: 128 additions on the tensor cores of one unit each, three roundings a block, one addition a block."""
import numpy as np
import pytest
import torch
from helpers import to_np
from test_matmul8_gpu import Operand, expected

import paper_2110_15032_b200 as sbp

pytestmark = pytest.mark.gpu
F32, B = torch.float32, sbp.B


# the operands exchanged, a few rows; tiles of 32 columns; the pair form; operands by plain loads
@pytest.mark.parametrize("m,n,kk", [(16, 512, 1024), (300, 200, 512), (2600, 2300, 400), (70, 300, 333)])
@pytest.mark.parametrize("xt,wt", [(False, True), (False, False), (True, False)])
@pytest.mark.parametrize("power", [110, -110, 125, -125])
@pytest.mark.parametrize("small", [False, True])
def test_scales_that_only_their_product_brings_back(m, n, kk, xt, wt, power, small):
    rng = np.random.default_rng(m + power + 200)
    x, w = Operand(m, kk, B, 1, xt, rng), Operand(n, kk, B, 1, wt, rng)
    for op, e in ((x, power), (w, -power)):
        if small:                                  # values down to the smallest, 2^-9
            op.values.locals[0].copy_((op.values.locals[0].float() / 448 * 2.0 ** -5).to(torch.float8_e4m3fn))
        s = op.scales.locals[0]
        s.copy_((1.0 + torch.from_numpy(rng.random(tuple(s.shape))).float().cuda()) * 2.0 ** e)
    y = sbp.empty_global((m, n), F32, B, 1)
    sbp.sbp_matmul8(x.values, x.scales, w.values, w.scales, y)
    torch.cuda.synchronize()
    want, mag = expected(x, w, "whole", 1, m, n)[0]
    got = to_np(y.locals[0]).astype(np.float64)
    by = (128 * 2.0 ** -23 + (-(-kk // 128) + 5) * 2.0 ** -24) * mag + 2.0 ** -24 * np.abs(want) + 1e-38
    bad = ~(np.abs(got - want) <= by)
    assert not bad.any(), f"{int(bad.sum())} of {bad.size}, {np.nanmax(np.abs(got - want) / by)} of the bound, {int((~np.isfinite(got)).sum())} not finite"
