"""The sign of zero in 8-bit blocks: -0 stays -0 whatever else its block, its row or its tile holds."""
import pytest
import torch

import paper_2110_15032_b200 as sbp

pytestmark = pytest.mark.gpu
F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
TILES, TRANS = sbp.SBP_QUANT_TILES, sbp.SBP_TRANS_X


@pytest.mark.parametrize("flags", [0, TILES, TRANS, TILES | TRANS])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(9, 256), (130, 257)])
@pytest.mark.parametrize("other", [1.0, float("nan"), float("inf")])
def test_zeros_keep_their_sign(flags, dtype, rows, cols, other):
    x = torch.zeros(rows, cols, dtype=dtype, device="cuda")
    x[:, ::3] = -0.0
    x[4, 6] = other
    shape = (cols, rows) if flags & TRANS else (rows, cols)
    q = sbp.empty_global(shape, E4M3, sbp.B, 1)
    s = sbp.empty_global(sbp.sbp_scales_shape(shape, sbp.B, 1, flags & TILES), F32, sbp.B, 1)
    sbp.sbp_quantize8(sbp.SbpTensor((rows, cols), dtype, sbp.B, [x]), q, s, flags)
    got = [q.locals[0].view(torch.uint8)]
    if not flags:
        y = sbp.empty_global(shape, dtype, sbp.B, 1)
        sbp.sbp_gelu_save8(sbp.SbpTensor((rows, cols), dtype, sbp.B, [x]), y, q, s)
        got.append(q.locals[0].view(torch.uint8))
    torch.cuda.synchronize()
    want = torch.zeros(rows, cols, dtype=torch.uint8, device="cuda")
    want[:, ::3] = 0x80
    for g in got:
        g = (g.t() if flags & TRANS else g).clone()
        g[4, 6] = 0x80                               # what the other element became is not asked here
        assert torch.equal(g, want)
