"""A wait that runs out inside an 8-bit product whose contraction is shared by a cluster: one of the warps that keep the accumulators gives up
while the others see all their blocks.  The kernel ends, the error is reported once and the same product runs as before."""
import numpy as np
import pytest
import torch
from helpers import to_np
from test_matmul8_gpu import Operand, expected

import paper_2110_15032_b200 as sbp

pytestmark = pytest.mark.gpu
F32, B = torch.float32, sbp.B


# tiles of 32 and 128 columns, the exchanged operands, and operands by plain loads
@pytest.mark.parametrize("m,n,kk,pitch", [(300, 200, 2048, 0), (300, 1000, 4096, 0), (9, 700, 4096, 0), (16, 1000, 2001, 1), (300, 200, 2049, 0)])
def test_a_warp_that_gives_up_ends_the_kernel(m, n, kk, pitch):
    rng = np.random.default_rng(m + n)
    x, w = Operand(m, kk, B, 1, False, rng, True, pitch), Operand(n, kk, B, 1, True, rng, True, pitch)
    want = expected(x, w, "whole", 1, m, n)[0][0]
    y = sbp.empty_global((m, n), F32, B, 1)
    args = (x.values, x.scales, w.values, w.scales, y)
    for warp in (0, 3, 7):
        sbp.sbp_selftest_matmul8_wait_timeout(*args, warp)
        torch.cuda.synchronize()
        with pytest.raises(sbp.SbpError) as e:
            sbp.sbp_check_device_errors()
        assert e.value.name == "SBP_ERR_TIMEOUT"
        sbp.sbp_check_device_errors()
        y.locals[0].fill_(float("nan"))
        sbp.sbp_matmul8(*args)
        torch.cuda.synchronize()
        sbp.sbp_check_device_errors()
        assert np.array_equal(to_np(y.locals[0]).astype(np.float64), want)


def test_products_without_a_shared_contraction_refuse_it():
    rng = np.random.default_rng(1)
    x, w = Operand(16, 128, B, 1, False, rng, True), Operand(16, 128, B, 1, True, rng, True)
    args = (x.values, x.scales, w.values, w.scales, sbp.empty_global((16, 16), F32, B, 1))
    for warp, name in ((0, "SBP_ERR_UNSUPPORTED"), (8, "SBP_ERR_INVALID_ARG"), (-1, "SBP_ERR_INVALID_ARG")):
        with pytest.raises(sbp.SbpError) as e:
            sbp.sbp_selftest_matmul8_wait_timeout(*args, warp)
        assert e.value.name == name
