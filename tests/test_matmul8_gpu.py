"""Products of 8-bit blocks against the oracle in fp64.

Tolerance: a block's 128 products are summed on the tensor cores, whose every addition is off by at most one unit in the last place of
fp32 (2^-23) of a partial sum; a scaled block sum has three roundings (product of scales, product, addition) and there are as many additions as blocks:
    |error| <= (128 * 2^-23 + (blocks + 4) 2^-24) * sum |x w| scales   + half a step of the result's type.
Whole numbers whose sums stay below 2^24 are exact in fp32 whatever the order."""
import numpy as np
import pytest
import torch
from helpers import make_global, to_np

import paper_2110_15032_b200 as sbp
from oracle import sbp_oracle as O

pytestmark = pytest.mark.gpu
F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
S0, S1, B, P = sbp.S(0), sbp.S(1), sbp.B, sbp.P_SUM
TILES = sbp.SBP_QUANT_TILES


def np8(t):
    return t.detach().cpu().float().numpy().astype(np.float64)


class Operand:
    """A stored 8-bit operand [rows, k] with random values and scales, its local tensors laid out as asked."""

    def __init__(self, rows, kk, sig, k, tiles, rng, whole=False, pitch=0, offset=0):
        self.shape, self.sig, self.k, self.tiles = (rows, kk), sig, k, tiles
        locs, scs = [], []
        sshape = sbp.sbp_scales_shape((rows, kk), sig, k, TILES if tiles else 0)
        for r in range(k):
            if sig is B and r:
                locs.append(locs[0])
                scs.append(scs[0])
                continue
            shp = sbp.sbp_local_shape((rows, kk), sig, k, r, E4M3)
            if whole:
                v = torch.from_numpy(rng.integers(-4, 5, shp).astype(np.float32))
                s = torch.from_numpy(np.exp2(rng.integers(-2, 1, sbp.sbp_local_shape(sshape, sig, k, r))).astype(np.float32))
            else:
                v = torch.from_numpy(rng.normal(0, 40, shp).astype(np.float32)).clamp(-448, 448)
                s = torch.from_numpy((np.exp(rng.normal(0, 1, sbp.sbp_local_shape(sshape, sig, k, r))) / 40).astype(np.float32))
            ld = max(1, shp[1] + pitch)
            raw = torch.zeros(offset + max(1, shp[0]) * ld + 16, dtype=torch.uint8, device="cuda").fill_(0x7F).view(E4M3)      # NaN around it
            t = raw[offset:offset + shp[0] * ld].view(shp[0], ld)[:, :shp[1]]
            t.copy_(v.cuda().to(E4M3))
            locs.append(t)
            scs.append(s.cuda())
        self.values = sbp.SbpTensor((rows, kk), E4M3, sig, locs)
        self.scales = sbp.SbpTensor(sshape, F32, sig, scs)

    def dense(self, r):
        return O.dequantize8(np8(self.values.locals[r]), to_np(self.scales.locals[r]), self.tiles)


ROWS = {   # signatures of x, of stored w, of y
    "rows": (S0, B, S0), "columns": (B, S0, S1), "partial": (S1, S1, P), "fused_b": (S1, S1, B), "fused_s0": (S1, S1, S0),
    "fused_s1": (S1, S1, S1), "whole": (B, B, B), "px": (P, B, P), "pw": (B, P, P),
}


def expected(x, w, sig, k, m, n):
    """Per shard: the exact result and the sum of magnitudes."""
    def local(r):
        a, b = x.dense(r), w.dense(r)
        return a @ b.T, np.abs(a) @ np.abs(b).T
    parts = [local(r) for r in range(k)]
    if not sig.startswith("fused"):
        return parts
    whole, mag = sum(p[0] for p in parts), sum(p[1] for p in parts)
    ysig = ROWS[sig][2]
    out = []
    for r in range(k):
        if ysig is B:
            out.append((whole, mag))
        else:
            shp = sbp.sbp_local_shape((m, n), ysig, k, r)
            start = sum(sbp.sbp_local_shape((m, n), ysig, k, i)[ysig.axis] for i in range(r))
            at = (slice(start, start + shp[0]), slice(None)) if ysig.axis == 0 else (slice(None), slice(start, start + shp[1]))
            out.append((whole[at], mag[at]))
    return out


def run(m, n, kk, k, sig, out, xt, wt, seed, whole=False, xpitch=0, wpitch=0, xoff=0, woff=0):
    rng = np.random.default_rng(seed)
    sx, sw, sy = ROWS[sig]
    x = Operand(m, kk, sx, k, xt, rng, whole, xpitch, xoff)
    w = Operand(n, kk, sw, k, wt, rng, whole, wpitch, woff)
    y = sbp.empty_global((m, n), out, sy, k)
    sbp.sbp_matmul8(x.values, x.scales, w.values, w.scales, y)
    torch.cuda.synchronize()
    for r, (want, mag) in enumerate(expected(x, w, sig, k, m, n)):
        got = to_np(y.locals[r]).astype(np.float64)
        if whole:
            assert out is F32 and np.array_equal(got, want), f"shard {r}: {np.argwhere(got != want)[:4]}"
        else:
            by = (128 * 2.0 ** -23 + (-(-kk // 128) + k + 4) * 2.0 ** -24) * mag
            half = 2.0 ** -8 if out is BF16 else 2.0 ** -24
            by = by * (1 + half) + half * np.abs(want) + 1e-38
            bad = ~(np.abs(got - want) <= by)
            assert not bad.any(), f"shard {r}: {int(bad.sum())} of {bad.size}, first {np.argwhere(bad)[:3]}, {np.nanmax(np.abs(got - want) / by)}"
    return x, w, y


# few rows or columns (the operands exchanged or not), one block and less, edges of tiles, lengths of one
@pytest.mark.parametrize("m,n,kk", [(1, 1, 1), (1, 256, 128), (16, 512, 1024), (17, 300, 400), (33, 130, 272), (64, 1000, 4096), (200, 16, 512),
                                    (130, 33, 640), (128, 128, 128), (129, 257, 144), (300, 200, 2048), (65, 65, 16), (257, 511, 48), (1000, 64, 256)])
@pytest.mark.parametrize("xt,wt", [(False, True), (False, False), (True, True), (True, False)])
def test_one_device_whole_numbers(m, n, kk, xt, wt):
    run(m, n, kk, 1, "whole", F32, xt, wt, m * n + kk, whole=True)


@pytest.mark.parametrize("sig", list(ROWS))
@pytest.mark.parametrize("m,n,kk", [(100, 260, 1040), (9, 700, 528), (400, 20, 272), (300, 600, 400)])
@pytest.mark.parametrize("out", [F32, BF16])
def test_signatures(sig, m, n, kk, out):
    run(m, n, kk, 3, sig, out, False, True, m + n + kk)
    if out is F32:
        run(m, n, kk, 3, sig, out, False, True, m + n, whole=True)


@pytest.mark.parametrize("sig", ["rows", "columns", "fused_b", "fused_s0", "fused_s1", "whole"])
@pytest.mark.parametrize("xt,wt", [(False, True), (False, False)])
def test_the_pair_form(sig, xt, wt):
    """Enough tiles of 256 x 256 for the persistent form, several a pair, ragged at every end."""
    run(2600, 2300, 400, 2, sig, F32, xt, wt, 77, whole=True)
    run(2600, 2300, 656, 2, sig, BF16, xt, wt, 78)


@pytest.mark.parametrize("m,n,kk", [(5, 300, 129), (200, 260, 333), (70, 70, 1), (16, 1000, 127), (300, 300, 1001)])
@pytest.mark.parametrize("sig", ["columns", "fused_b", "rows"])
def test_rows_that_the_copy_engine_does_not_take(m, n, kk, sig):
    run(m, n, kk, 2, sig, F32, False, True, kk, whole=True)
    run(m, n, kk, 2, sig, BF16, False, False, kk + 1)


@pytest.mark.parametrize("xpitch,wpitch,xoff,woff", [(16, 32, 16, 48), (3, 0, 0, 0), (0, 5, 1, 0), (0, 0, 0, 7), (13, 1, 2, 3)])
def test_windows_and_odd_bases(xpitch, wpitch, xoff, woff):
    """What lies around the operands is NaN."""
    run(150, 200, 304, 2, "columns", F32, False, True, 5, True, xpitch, wpitch, xoff, woff)
    run(7, 200, 304, 2, "columns", F32, False, True, 6, True, xpitch, wpitch, xoff, woff)


def test_result_windows_and_replicas():
    rng = np.random.default_rng(3)
    for m, n in ((40, 300), (300, 150), (9, 500)):
        x, w = Operand(m, 256, B, 2, False, rng, True), Operand(n, 256, B, 2, True, rng, True)
        want = expected(x, w, "whole", 2, m, n)[0][0]
        for dtype, skip, extra in ((F32, 4, 8), (F32, 3, 9), (BF16, 5, 7)):
            bufs = [torch.full((m, n + extra), 7.0, dtype=dtype, device="cuda") for _ in range(2)]
            y = sbp.SbpTensor((m, n), dtype, B, [b[:, skip:skip + n] for b in bufs])
            sbp.sbp_matmul8(x.values, x.scales, w.values, w.scales, y)
            torch.cuda.synchronize()
            for b in bufs:
                got = to_np(b[:, skip:skip + n].contiguous()).astype(np.float64)
                assert np.array_equal(got, to_np(torch.from_numpy(want).float().to(dtype)))
                assert (b[:, :skip] == 7.0).all() and (b[:, skip + n:] == 7.0).all()


def test_nothing_to_contract_and_nothing_to_compute():
    rng = np.random.default_rng(4)
    for m, n in ((5, 300), (300, 300)):
        x, w = Operand(m, 0, B, 1, False, rng), Operand(n, 0, B, 1, True, rng)
        y = sbp.empty_global((m, n), F32, B, 1)
        sbp.sbp_matmul8(x.values, x.scales, w.values, w.scales, y)
        torch.cuda.synchronize()
        assert (y.locals[0] == 0).all()
    x, w = Operand(0, 128, B, 1, False, rng), Operand(9, 128, B, 1, True, rng)
    before = sbp.sbp_launch_count()
    sbp.sbp_matmul8(x.values, x.scales, w.values, w.scales, sbp.empty_global((0, 9), F32, B, 1))
    assert sbp.sbp_launch_count() == before
    # more devices than rows: some hold none
    run(2, 300, 256, 4, "rows", F32, False, True, 9, whole=True)
    run(300, 3, 256, 5, "columns", F32, False, True, 9, whole=True)
    run(30, 40, 3, 5, "fused_b", F32, False, True, 9, whole=True)          # and some none of the contraction


@pytest.mark.parametrize("m,n", [(3, 400), (200, 300), (2600, 2300)])
def test_nan_stays_in_its_row_and_column(m, n):
    rng = np.random.default_rng(5)
    x, w = Operand(m, 384, B, 1, False, rng, True), Operand(n, 384, B, 1, True, rng, True)
    want = expected(x, w, "whole", 1, m, n)[0][0]
    x.values.locals[0].view(torch.uint8)[1, 200] = 0x7F
    w.values.locals[0].view(torch.uint8)[37, 3] = 0xFF
    y = sbp.empty_global((m, n), F32, B, 1)
    sbp.sbp_matmul8(x.values, x.scales, w.values, w.scales, y)
    torch.cuda.synchronize()
    got = to_np(y.locals[0]).astype(np.float64)
    assert np.isnan(got[1]).all() and np.isnan(got[:, 37]).all()
    got[1], got[:, 37] = want[1], want[:, 37]
    assert np.array_equal(got, want)


def test_same_bits_every_time_on_streams_and_in_a_graph():
    rng = np.random.default_rng(6)
    cases = []
    for m, n, kk in ((16, 1024, 2048), (300, 500, 1024), (2600, 2300, 512)):
        x, w = Operand(m, kk, B, 1, False, rng), Operand(n, kk, B, 1, True, rng)
        y = sbp.empty_global((m, n), BF16, B, 1)
        sbp.sbp_matmul8(x.values, x.scales, w.values, w.scales, y)
        torch.cuda.synchronize()
        cases.append((x, w, y, y.locals[0].clone()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for x, w, y, _ in cases:
            sbp.sbp_matmul8(x.values, x.scales, w.values, w.scales, y)
    for _ in range(3):
        for c in cases:
            c[2].locals[0].fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(c[2].locals[0], c[3]) for c in cases)
    streams = [torch.cuda.Stream() for _ in cases]
    for c in cases:
        c[2].locals[0].fill_(float("nan"))
    torch.cuda.synchronize()
    for c, st in zip(cases, streams):
        sbp.sbp_matmul8(c[0].values, c[0].scales, c[1].values, c[1].scales, c[2], stream=st)
    torch.cuda.synchronize()
    assert all(torch.equal(c[2].locals[0], c[3]) for c in cases)
