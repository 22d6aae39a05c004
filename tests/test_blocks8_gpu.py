"""8-bit blocks: quantisation in its four forms is exact, element for element and scale for scale; GeLU with its 8-bit checkpoint and
the gradient through it, against the oracle in fp64.

Tolerance of GeLU: 2^-20 relative from the error function, z^2 u from rounding the exponent z^2 / 2 (u = 2^-24), half a step of
the result's type, and fp32's smallest normal number."""
import numpy as np
import pytest
import torch
from helpers import make_global, split_cpu, to_np

import paper_2110_15032_b200 as sbp
import sbp_datagen as dg
from oracle import sbp_oracle as O

pytestmark = pytest.mark.gpu
F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
S0, S1, B = sbp.S(0), sbp.S(1), sbp.B
TILES, TRANS = sbp.SBP_QUANT_TILES, sbp.SBP_TRANS_X
U = 2.0 ** -24


def half_step(dtype):
    return 2.0 ** -8 if dtype == BF16 else 2.0 ** -24


def np8(t):
    return t.detach().cpu().float().numpy().astype(np.float64)


def spread(shape, seed, dtype):
    """Blocks of very different sizes, exact zeros, whole blocks of zeros."""
    x = dg.normal(seed, 0, shape, 0.0, 1.0, F32).reshape(-1, shape[-1])
    x = x * torch.exp2(torch.floor(dg.normal(seed, 1, (x.shape[0], 1), 0.0, 12.0, F32)))
    x[:, ::7] *= 2.0 ** -9
    x[:, 1::11] = 0.0
    if x.shape[0] > 2:
        x[2] = 0.0
    return x.reshape(shape).to(dtype)


def out8(shape, sig, k, flags=0, alias=False):
    q = sbp.empty_global(shape, E4M3, sig, k, alias_replicas=alias)
    s = sbp.empty_global(sbp.sbp_scales_shape(shape, sig, k, flags & TILES), F32, sig, k, alias_replicas=alias)
    return q, s


def same_blocks(x, q, s, flags, what):
    """One local tensor, a matrix."""
    want_q, want_s = O.quantize8(x.T if flags & TRANS else x, bool(flags & TILES))
    assert np.array_equal(to_np(s).astype(np.float64).reshape(want_s.shape), want_s), f"scales {what}"
    got = np8(q).reshape(want_q.shape)
    assert np.array_equal(got, want_q, equal_nan=True), f"values {what}: {np.argwhere(~((got == want_q) | (np.isnan(got) & np.isnan(want_q))))[:3]}"


SIZES = [(1, 1), (3, 128), (200, 256), (130, 257), (5, 130), (64, 2048), (33, 4100), (300, 129), (2, 9000), (1, 16), (127, 8), (129, 1000)]


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("flags", [0, TILES, TRANS, TILES | TRANS])
@pytest.mark.parametrize("dtype,k,axis", [(BF16, 3, 0), (F32, 2, 1), (BF16, 1, 0)])
def test_quantize_is_exact(rows, cols, flags, dtype, k, axis):
    X = spread((rows, cols), rows + cols, dtype)
    sig = sbp.S(axis)
    x = make_global(split_cpu(X, sig, k), (rows, cols), dtype, sig)
    shape, qsig = ((cols, rows), sbp.S(1 - axis)) if flags & TRANS else ((rows, cols), sig)
    q, s = out8(shape, qsig, k, flags)
    sbp.sbp_quantize8(x, q, s, flags)
    torch.cuda.synchronize()
    for r in range(k):
        if x.locals[r].numel():
            same_blocks(to_np(x.locals[r]).astype(np.float64), q.locals[r], s.locals[r], flags, f"shard {r}")


@pytest.mark.parametrize("flags", [0, TILES, TRANS, TILES | TRANS])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_quantize_at_the_ends_of_the_range(flags, dtype):
    """Infinities, NaN, the largest numbers, subnormal ones, and every number near a tie."""
    X = torch.zeros(140, 300)
    X[0, :5] = torch.tensor([float("inf"), 1.0, -3.0, float("nan"), float("-inf")])
    X[1, 0], X[1, 1] = torch.finfo(dtype).max, 1.0
    X[2, 0], X[2, 1], X[2, 2] = 2.0 ** -133, -(2.0 ** -130), 2.0 ** -127
    X[3, 128:256] = float("nan")
    X[4, :128] = torch.arange(128) * 3.5
    X[5, :120] = torch.arange(120, dtype=torch.uint8).view(E4M3).float() * (1 + 2.0 ** -4)
    X[6, 0], X[6, 1] = 448.0 * 2.0 ** -126, 449.0 * 2.0 ** -126
    X[7, :64] = 448.0
    X[8, :64] = 448.0 * (1 + 2.0 ** -7)
    X[139, 299] = -1e-30
    X = X.to(dtype)
    x = make_global([X], (140, 300), dtype, S0)
    shape = (300, 140) if flags & TRANS else (140, 300)
    q, s = out8(shape, S0 if not flags & TRANS else S1, 1, flags)
    sbp.sbp_quantize8(x, q, s, flags)
    torch.cuda.synchronize()
    same_blocks(to_np(X).astype(np.float64), q.locals[0], s.locals[0], flags, "")


@pytest.mark.parametrize("axis", [0, 1, 2])
def test_quantize_of_three_axes_and_replicas(axis):
    X = spread((4, 5, 300), 9, BF16)
    sig = sbp.S(axis)
    x = make_global(split_cpu(X, sig, 2), (4, 5, 300), BF16, sig)
    q, s = out8((4, 5, 300), sig, 2)
    sbp.sbp_quantize8(x, q, s)
    torch.cuda.synchronize()
    for r in range(2):
        same_blocks(to_np(x.locals[r]).astype(np.float64).reshape(-1, x.locals[r].shape[-1]), q.locals[r], s.locals[r], 0, f"shard {r}")
    xb = sbp.SbpTensor((4, 5, 300), BF16, B, [X.cuda()] * 2)
    for alias in (False, True):
        qb, sb = out8((4, 5, 300), B, 2, alias=alias)
        sbp.sbp_quantize8(xb, qb, sb)
        torch.cuda.synchronize()
        for r in range(2):
            same_blocks(to_np(X).astype(np.float64).reshape(-1, 300), qb.locals[r], sb.locals[r], 0, f"replica {r}")


@pytest.mark.parametrize("flags", [0, TILES, TRANS, TILES | TRANS])
@pytest.mark.parametrize("skip,extra", [(16, 32), (1, 5)])
def test_quantize_windows(flags, skip, extra):
    rows, cols = 70, 272
    buf = torch.zeros(rows, cols + extra, dtype=BF16, device="cuda")
    x = buf[:, skip if skip < extra else 0:][:, :cols]
    x.copy_(spread((rows, cols), 12, BF16))
    shape = (cols, rows) if flags & TRANS else (rows, cols)
    into = torch.zeros(shape[0], shape[1] + extra, dtype=torch.uint8, device="cuda").fill_(0x55).view(E4M3)
    v = into[:, skip:][:, :shape[1]] if skip < extra else into[:, :shape[1]]
    q = sbp.SbpTensor(shape, E4M3, S0, [v])
    s = sbp.empty_global(sbp.sbp_scales_shape(shape, S0, 1, flags & TILES), F32, S0, 1)
    sig = S1 if flags & TRANS else S0
    sbp.sbp_quantize8(sbp.SbpTensor((rows, cols), BF16, sig, [x]), q, s, flags)
    torch.cuda.synchronize()
    same_blocks(to_np(x.contiguous()).astype(np.float64), v.contiguous(), s.locals[0], flags, "")
    raw = into.view(torch.uint8)
    assert (raw[:, :skip] == 0x55).all() and (raw[:, skip + shape[1]:] == 0x55).all()


def gelu_bound(z, want, dtype):
    return np.abs(want) * (2.0 ** -20 + z * z * U) * (1 + half_step(dtype)) + half_step(dtype) * np.abs(want) + 2.0 ** -126


def close(got, want, bound, what):
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.size}, {np.nanmax(np.abs(got - want) / bound):.2f} of the bound"


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("zt,yt,k,axis", [(BF16, BF16, 2, 1), (F32, F32, 3, 0), (F32, BF16, 1, 0), (BF16, F32, 2, 0)])
def test_gelu_and_its_checkpoint(rows, cols, zt, yt, k, axis):
    Z = dg.normal(rows * cols, 0, (rows, cols), 0.0, 2.5, zt)
    sig = sbp.S(axis)
    z = make_global(split_cpu(Z, sig, k), (rows, cols), zt, sig)
    y = sbp.empty_global((rows, cols), yt, sig, k)
    q, s = out8((rows, cols), sig, k)
    sbp.sbp_gelu_save8(z, y, q, s)
    torch.cuda.synchronize()
    for r in range(k):
        if not z.locals[r].numel():
            continue
        v = to_np(z.locals[r]).astype(np.float64)
        same_blocks(v, q.locals[r], s.locals[r], 0, f"shard {r}")
        want = O.gelu_from_erfc(v)
        close(to_np(y.locals[r]).astype(np.float64), want, gelu_bound(v, want, yt), f"y {r}")


def test_gelu_of_every_bf16():
    Z = torch.arange(65536, dtype=torch.int32).to(torch.uint16).view(BF16).reshape(512, 128)
    Z = torch.where(torch.isfinite(Z.float()), Z, torch.zeros_like(Z))
    z = make_global([Z], (512, 128), BF16, S0)
    for yt in (BF16, F32):
        y = sbp.empty_global((512, 128), yt, S0, 1)
        q, s = out8((512, 128), S0, 1)
        sbp.sbp_gelu_save8(z, y, q, s)
        torch.cuda.synchronize()
        v = to_np(Z).astype(np.float64)
        want = O.gelu_from_erfc(v)
        close(to_np(y.locals[0]).astype(np.float64), want, gelu_bound(v, want, yt), "y")


def test_gelu_of_what_is_not_finite():
    Z = torch.tensor([[float("inf"), float("nan"), -1.0, 2.0]])
    z = make_global([Z], (1, 4), F32, S0)
    y = sbp.empty_global((1, 4), F32, S0, 1)
    q, s = out8((1, 4), S0, 1)
    sbp.sbp_gelu_save8(z, y, q, s)
    torch.cuda.synchronize()
    got = y.locals[0].cpu()[0]
    assert got[0] == float("inf") and torch.isnan(got[1]) and abs(got[3].item() - 1.9544997) < 1e-6
    assert torch.isnan(q.locals[0].float()[0, :2]).all() and q.locals[0].float()[0, 2:].tolist() == [-128.0, 256.0]      # 2 <= 448 * 2^-7


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dyt,dzt,k,axis", [(BF16, BF16, 2, 1), (F32, F32, 3, 0), (F32, BF16, 1, 0), (BF16, F32, 2, 0)])
def test_gelu_gradient_from_the_checkpoint(rows, cols, dyt, dzt, k, axis):
    sig = sbp.S(axis)
    Z, DY = dg.normal(rows, 0, (rows, cols), 0.0, 2.5, F32), dg.normal(rows, 1, (rows, cols), 0.0, 1.0, dyt)
    z = make_global(split_cpu(Z, sig, k), (rows, cols), F32, sig)
    q, s = out8((rows, cols), sig, k)
    sbp.sbp_quantize8(z, q, s)
    if rows > 1:
        for t in s.locals:
            t *= 1.1                                   # any fp32 scale
    dy = make_global(split_cpu(DY, sig, k), (rows, cols), dyt, sig)
    dz = sbp.empty_global((rows, cols), dzt, sig, k)
    sbp.sbp_gelu_save8_backward(q, s, dy, dz)
    torch.cuda.synchronize()
    for r in range(k):
        if not dy.locals[r].numel():
            continue
        v, d = O.dequantize8(np8(q.locals[r]), to_np(s.locals[r])), to_np(dy.locals[r]).astype(np.float64)
        want = d * O.gelu_slope(v)
        # the two terms are each right to 2^-20 and what z^2 brings; value times scale is rounded once: slope' <= 0.8 per unit of z
        terms = 0.5 * O._erfc(-v / np.sqrt(2)) + np.abs(v) * np.exp(-0.5 * v * v) / np.sqrt(2 * np.pi)
        by = np.abs(d) * (terms * (2.0 ** -20 + 2 * v * v * U) + 0.8 * np.abs(v) * U)
        by = by * (1 + half_step(dzt)) + half_step(dzt) * np.abs(want) + 2.0 ** -126
        close(to_np(dz.locals[r]).astype(np.float64), want, by, f"grad_z {r}")


def test_gradient_at_every_e4m3_number():
    """Both zeros, the subnormal numbers, NaN, under small and large scales."""
    codes = torch.arange(256, dtype=torch.uint8).reshape(1, 256).repeat(6, 1)
    scales = torch.tensor([2.0 ** -20, 2.0 ** -8, 0.013, 1.0, 3.7, 2.0 ** 60]).reshape(6, 1).repeat(1, 2)
    q, s = make_global([codes.view(E4M3)], (6, 256), E4M3, S0), make_global([scales], (6, 2), F32, S0)
    dy = make_global([torch.ones(6, 256)], (6, 256), F32, S0)
    dz = sbp.empty_global((6, 256), F32, S0, 1)
    sbp.sbp_gelu_save8_backward(q, s, dy, dz)
    torch.cuda.synchronize()
    got = to_np(dz.locals[0]).astype(np.float64)
    nan = np.isnan(codes.view(E4M3).float().numpy())
    assert nan.sum() == 12 and np.array_equal(np.isnan(got), nan)
    v = O.dequantize8(codes.view(E4M3).float().numpy().astype(np.float64), scales.numpy())
    v = np.where(nan, 0.0, v)
    want = O.gelu_slope(np.clip(v, -40, 40))               # beyond, the slope is 0 or 1
    terms = 0.5 * O._erfc(-v / np.sqrt(2)) + np.abs(np.clip(v, -40, 40)) * np.exp(-0.5 * v * v) / np.sqrt(2 * np.pi)
    by = terms * (2.0 ** -20 + 2 * np.minimum(v * v, 400) * U) + 0.8 * np.minimum(np.abs(v), 40) * U + U * np.abs(want) + 2.0 ** -126
    close(np.where(nan, want, got), want, by, "slope")


def test_gradient_against_differences_of_gelu():
    """With a checkpoint that holds z exactly (e4m3 numbers), the gradient is that of GeLU at z."""
    Z = torch.arange(-24, 24, dtype=F32).reshape(1, 48) / 8
    z = make_global([Z], (1, 48), F32, S0)
    q, s = out8((1, 48), S0, 1)
    y, dz = sbp.empty_global((1, 48), F32, S0, 1), sbp.empty_global((1, 48), F32, S0, 1)
    sbp.sbp_gelu_save8(z, y, q, s)
    sbp.sbp_gelu_save8_backward(q, s, make_global([torch.ones(1, 48)], (1, 48), F32, S0), dz)
    torch.cuda.synchronize()
    v = O.dequantize8(np8(q.locals[0]), to_np(s.locals[0]))
    h = 1e-6
    diff = (O.gelu_from_erfc(v + h) - O.gelu_from_erfc(v - h)) / (2 * h)
    assert np.max(np.abs(to_np(dz.locals[0]) - diff)) < 1e-6


def test_empty_tensors_launch_nothing():
    x, before = sbp.empty_global((0, 64), F32, S0, 2), sbp.sbp_launch_count()
    q, s = out8((0, 64), S0, 2)
    sbp.sbp_quantize8(x, q, s)
    sbp.sbp_gelu_save8(x, x, q, s)
    sbp.sbp_gelu_save8_backward(q, s, x, x)
    assert sbp.sbp_launch_count() == before
