"""What the library's choice of a form for an 8-bit product rests on: the price of a block in each form as it is built."""
import numpy as np
import pytest
import torch
from test_matmul8_gpu import Operand

import paper_2110_15032_b200 as sbp

pytestmark = pytest.mark.gpu
FORMS = [(c, s, e, y) for c in (256, 128, 64, 32, 16) for s in (1, 2, 4, 8) for e in (0, 1) for y in (0, 1)]


def chosen(m, n, kk, wt):
    rng = np.random.default_rng(1)
    x, w = Operand(m, kk, sbp.B, 1, False, rng), Operand(n, kk, sbp.B, 1, wt, rng)
    count = lambda: {f: sbp.sbp_matmul8_form_launches(f[0], f[1], f[2], 1, f[3]) for f in FORMS}
    before = count()
    sbp.sbp_matmul8(x.values, x.scales, w.values, w.scales, sbp.empty_global((m, n), torch.bfloat16, sbp.B, 1))
    torch.cuda.synchronize()
    return [f for f, c in count().items() if c != before[f]]


@pytest.mark.parametrize("m,n,kk", [(1926, 2904, 6400), (4096, 3000, 4096)])
def test_large_products_with_a_scale_for_each_column_take_pairs(m, n, kk):
    """1926 x 2904 x 6400: 94 us in the pair form, 128 in tiles of 128 columns that two CTAs share."""
    assert chosen(m, n, kk, False) == [(256, 1, 0, 1)]


@pytest.mark.parametrize("wt", [True, False])
@pytest.mark.parametrize("m,n,kk", [(512, 512, 8192), (1472, 336, 5104), (409, 288, 4256)])
def test_no_more_clusters_than_the_device_holds_at_once(m, n, kk, wt):
    """A contraction is shared to fill the device in one wave.  148 SMs have room for 33 clusters of four CTAs and 15 of eight, where a CTA takes an SM, and
    for 71 and 33 where two share one: 512 x 512 x 8192 as 16 clusters of eight took 21.8 us, as 32 clusters of four of the smaller ones 15.5."""
    (columns, splits, exchanged, _), = chosen(m, n, kk, wt)
    tiles = -(-(n if exchanged else m) // 128) * -(-(m if exchanged else n) // columns)
    held = {4: 71, 8: 33} if columns <= 32 else {4: 33, 8: 15}
    assert torch.cuda.get_device_properties(0).multi_processor_count != 148 or splits < 4 or tiles <= held[splits]
