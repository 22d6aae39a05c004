"""Every form of the 8-bit product, asked for and seen to have run: tiles of 16 to 256 columns, contractions shared by 1 to 8 CTAs, operands exchanged or
not, read by the copy engine or by plain loads, one scale for 128 columns or one for each -- on odd sizes, results whole numbers and exact."""
import itertools

import numpy as np
import pytest
import torch
from test_matmul8_gpu import run

import paper_2110_15032_b200 as sbp

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def exists(columns, copy_engine, scale_each):
    return scale_each or not (columns == 64 if copy_engine else columns == 16)


FORMS = [f for f in itertools.product((128, 64, 32, 16), (1, 2, 4, 8), (False, True), (False, True), (False, True)) if exists(f[0], f[3], f[4])]


@pytest.fixture(autouse=True)
def as_before():
    yield
    sbp.sbp_matmul8_set_form()


def forced(columns, splits, exchanged, copy_engine, scale_each, *args, **kw):
    sbp.sbp_matmul8_set_form(columns, splits, exchanged)
    before = sbp.sbp_matmul8_form_launches(columns, splits, exchanged, copy_engine, scale_each)
    run(*args, **kw)
    assert sbp.sbp_matmul8_form_launches(columns, splits, exchanged, copy_engine, scale_each) == before + 1


def layouts(exchanged, scale_each):
    """(x in tiles, w in tiles): the operand whose rows are the tile's columns has a scale for each, or one for 128."""
    return [(not scale_each, o) if exchanged else (o, not scale_each) for o in (False, True)]


@pytest.mark.parametrize("columns,splits,exchanged,copy_engine,scale_each", FORMS)
def test_edges_of_every_form(columns, splits, exchanged, copy_engine, scale_each):
    kk = 2304 + (16 if copy_engine else 5)             # 19 blocks, the last one short
    for xt, wt in layouts(exchanged, scale_each):
        for m, n in ((1, 1), (131, 257), (300, 33)):
            # (of one row the scales are the same either way, and count as a scale for each)
            forced(columns, splits, exchanged, copy_engine, scale_each or m == 1, m, n, kk, 1, "whole", F32, xt, wt, columns + m, whole=True)
        forced(columns, splits, exchanged, copy_engine, scale_each, 150, 270, kk, 1, "whole", BF16, xt, wt, columns)


# several groups, results with offsets, segments of unequal length that end inside a block (416 and 400 bytes: whole 16-byte pieces)
SIGS = ["rows", "columns", "partial", "fused_b", "fused_s0", "fused_s1"]


@pytest.mark.parametrize("sig", SIGS)
@pytest.mark.parametrize("columns,exchanged", [(c, e) for c in (128, 64, 32, 16) for e in (False, True)])
@pytest.mark.parametrize("splits", [1, 4])
def test_signatures_of_every_form(sig, columns, exchanged, splits):
    for copy_engine in (True, False):
        for scale_each in (True, False):
            if not exists(columns, copy_engine, scale_each):
                continue
            # parts that start inside a tile of 128 of the operand whose rows are the columns need a scale for each of them
            fused_offsets = sig == ("fused_s0" if exchanged else "fused_s1")
            m, n = (512, 300) if exchanged and not scale_each else (300, 512) if not scale_each else (301, 270)
            k = 2 if fused_offsets and not scale_each else 3
            kk = (k * 1248 if sig in ("partial", "fused_b", "fused_s0", "fused_s1") else 1264) + (0 if copy_engine else 1)
            for xt, wt in layouts(exchanged, scale_each):
                forced(columns, splits, exchanged, copy_engine, scale_each, m, n, kk, k, sig, F32, xt, wt, columns + m, whole=True)


@pytest.mark.parametrize("sig", SIGS + ["whole", "px", "pw"])
@pytest.mark.parametrize("scale_each", [False, True])
def test_the_pair_form_ran(sig, scale_each):
    """Several tiles a pair, ragged at every end; where shards are cut along the contraction, each holds 416 or 672 of it."""
    n = 2304 if not scale_each else 2300
    for kk, out, xt, whole in ((832, F32, False, True), (1344, BF16, True, False)):
        forced(256, 1, False, True, scale_each, 2600, n, kk, 2, sig, out, xt, not scale_each, 77 + kk, whole=whole)


def test_parts_that_start_inside_a_tile_of_scales():
    """One scale for 128 x 128, but the results' parts start between: a scale for each column, looked up in tiles."""
    forced(256, 1, False, True, True, 2600, 2300, 832, 2, "fused_s1", F32, False, True, 5, whole=True)
    for columns in (128, 64, 32, 16):
        forced(columns, 2, False, True, True, 300, 270, 1248, 3, "fused_s1", F32, True, True, 6, whole=True)
        forced(columns, 2, True, True, True, 300, 270, 1248, 3, "fused_s0", F32, True, True, 7, whole=True)


def test_the_library_chooses_the_pair_form_for_large_products():
    for wt in (True, False):
        before = sbp.sbp_matmul8_form_launches(256, 1, False, True, not wt)
        run(2600, 2300, 416, 1, "whole", F32, False, wt, 3, whole=True)
        assert sbp.sbp_matmul8_form_launches(256, 1, False, True, not wt) == before + 1


def test_a_form_that_a_product_cannot_run():
    total = lambda: [sbp.sbp_matmul8_form_launches(*f) for f in FORMS]
    sbp.sbp_matmul8_set_form(256, 1)                   # rows that the copy engine does not take
    before = total()
    run(70, 90, 333, 1, "whole", F32, False, True, 1, whole=True)
    assert sum(total()) == sum(before) + 1
    sbp.sbp_matmul8_set_form(64, 1)                    # one scale for 128 columns
    before = sbp.sbp_matmul8_form_launches(64, 1, False, True, False)
    run(70, 90, 336, 1, "whole", F32, False, True, 1, whole=True)
    assert sbp.sbp_matmul8_form_launches(64, 1, False, True, False) == before == 0
    forced_splits = sbp.sbp_matmul8_form_launches(128, 2, False, True, False)
    sbp.sbp_matmul8_set_form(128, 8)                   # five blocks: two shares
    run(70, 90, 592, 1, "whole", F32, False, True, 1, whole=True)
    assert sbp.sbp_matmul8_form_launches(128, 2, False, True, False) == forced_splits + 1
