"""Layer norm and the 8-bit path where order and offsets matter: inputs that the call before has just written and the call after writes again, with
no synchronisation in between, and tensors whose last elements lie beyond 2^31."""
import numpy as np
import pytest
import torch
from helpers import to_np

import paper_2110_15032_b200 as sbp
from oracle import sbp_oracle as O

pytestmark = pytest.mark.gpu
F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
S0, B, P = sbp.S(0), sbp.B, sbp.P_SUM
ROUNDS = 16


def one(t, k=1):
    return sbp.SbpTensor(tuple(t.shape), t.dtype, B, [t] * k)


def room(shape, dtype):
    return sbp.empty_global(shape, dtype, B, 1)


@pytest.mark.parametrize("m,h", [(64, 256), (700, 1024)])
def test_inputs_written_just_before(m, h):
    """Each round boxes other values into the same buffer and runs the chain norm, quantise, product, GeLU, its gradient, the norm's gradient; the
    rounds' results are those of the chain run alone, bit for bit."""
    torch.manual_seed(1)
    k = 2
    xs = [torch.randn(m, h, device="cuda").to(BF16) for _ in range(ROUNDS)]
    srcs = [sbp.SbpTensor((m, h), BF16, S0, [t.contiguous() for t in torch.tensor_split(x, k)]) for x in xs]
    w = one((torch.randn(h, h, device="cuda") * h ** -0.5).to(BF16))
    w8, w8s = room((h, h), E4M3), room(sbp.sbp_scales_shape((h, h), B, 1, sbp.SBP_QUANT_TILES), F32)
    sbp.sbp_quantize8(w, w8, w8s, sbp.SBP_QUANT_TILES)
    gamma = one(torch.rand(h, device="cuda") + 0.5)
    x, n, z, y, dz = (room((m, h), BF16) for _ in range(5))
    mean, rstd = room((m,), F32), room((m,), F32)
    n8, z8 = room((m, h), E4M3), room((m, h), E4M3)
    n8s, z8s = (room(sbp.sbp_scales_shape((m, h), B, 1), F32) for _ in range(2))
    ws = torch.empty(max(16, sbp.sbp_layer_norm_backward_workspace_bytes(x)), dtype=torch.uint8, device="cuda")
    xk = sbp.SbpTensor((m, h), BF16, B, [x.locals[0]] * k)

    def chain(src, outs):
        sbp.sbp_boxing(src, xk)
        sbp.sbp_layer_norm(x, gamma, None, n, mean, rstd)
        sbp.sbp_quantize8(n, n8, n8s)
        sbp.sbp_matmul8(n8, n8s, w8, w8s, z)
        sbp.sbp_gelu_save8(z, y, z8, z8s)
        sbp.sbp_gelu_save8_backward(z8, z8s, y, dz)
        sbp.sbp_layer_norm_backward(x, gamma, mean, rstd, dz, *outs, ws)

    def fresh():
        return room((m, h), BF16), room((h,), F32), room((h,), F32)
    alone = []
    for s in srcs:
        o = fresh()
        torch.cuda.synchronize()
        chain(s, o)
        torch.cuda.synchronize()
        alone.append(o)
    outs = [fresh() for _ in srcs]
    torch.cuda.synchronize()
    for s, o in zip(srcs, outs):
        chain(s, o)
    torch.cuda.synchronize()
    for i, (a, b) in enumerate(zip(alone, outs)):
        for u, v in zip(a, b):
            assert not torch.isnan(v.locals[0].float()).any() and torch.equal(u.locals[0], v.locals[0]), f"round {i}"


ROWS, COLS = 66000, 32768            # 2.16e9 elements


def test_blocks_beyond_32_bits():
    x = torch.zeros(ROWS, COLS, dtype=BF16, device="cuda")
    x[-3:] = torch.randn(3, COLS, device="cuda").to(BF16)
    q, s = torch.empty(ROWS, COLS, dtype=E4M3, device="cuda"), torch.empty(ROWS, COLS // 128, dtype=F32, device="cuda")
    y = torch.empty(ROWS, COLS, dtype=BF16, device="cuda")
    sbp.sbp_gelu_save8(one(x), one(y), one(q), one(s))
    torch.cuda.synchronize()
    tail = to_np(x[-3:]).astype(np.float64)
    want_q, want_s = O.quantize8(tail)
    assert np.array_equal(q[-3:].float().cpu().numpy(), want_q) and np.array_equal(to_np(s[-3:]), want_s)
    want = O.gelu_from_erfc(tail)
    assert np.all(np.abs(to_np(y[-3:]) - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -19 * np.abs(want) + 2.0 ** -126)
    q.view(torch.uint8).zero_()
    t = torch.empty(COLS, ROWS, dtype=E4M3, device="cuda")       # transposed: the last rows are the ends of the columns
    ts = torch.empty(COLS, -(-ROWS // 128), dtype=F32, device="cuda")
    sbp.sbp_quantize8(one(x), one(t), one(ts), sbp.SBP_TRANS_X)
    torch.cuda.synchronize()
    last = ROWS // 128 * 128                                     # the last block of a column holds rows from here on
    want_q, want_s = O.quantize8(to_np(x[last:, -256:]).astype(np.float64).T)
    assert np.array_equal(t[-256:, last:].float().cpu().numpy(), want_q) and np.array_equal(to_np(ts[-256:, -1:]), want_s)
    del q, s, t, ts
    # and back through the checkpoint
    q = torch.zeros(ROWS, COLS, dtype=E4M3, device="cuda")
    s = torch.ones(ROWS, COLS // 128, dtype=F32, device="cuda")
    q[-1] = 1.5
    sbp.sbp_gelu_save8_backward(one(q), one(s), one(x), one(y))
    torch.cuda.synchronize()
    want = tail[-1] * O.gelu_slope(1.5)
    assert np.all(np.abs(to_np(y[-1]) - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -19 * np.abs(want))


def test_layer_norm_beyond_32_bits():
    cols = 4096
    rows = ROWS * COLS // cols
    x = torch.zeros(rows, cols, dtype=BF16, device="cuda")
    x[-2:] = torch.randn(2, cols, device="cuda").to(BF16)
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    sbp.sbp_layer_norm(one(x), None, None, one(y), one(mean), one(rstd))
    torch.cuda.synchronize()
    want, m, r = O.layer_norm(to_np(x[-2:]).astype(np.float64), 1.0, 0.0, 1e-5)
    assert np.all(np.abs(to_np(y[-2:]) - want) <= 2.0 ** -8 * np.abs(want) + 1e-4)
    assert np.all(np.abs(to_np(mean[-2:]) - m) <= 1e-5) and np.all(np.abs(to_np(rstd[-2:]) - r) <= 1e-5 * r)
    gx, gg = torch.empty_like(x), torch.empty(cols, device="cuda")
    ws = torch.empty(sbp.sbp_layer_norm_backward_workspace_bytes(one(x)), dtype=torch.uint8, device="cuda")
    sbp.sbp_layer_norm_backward(one(x), None, one(mean), one(rstd), one(x), one(gx), one(gg), None, ws)
    torch.cuda.synchronize()
    tail = to_np(x[-2:]).astype(np.float64)
    dx, dg, _ = O.layer_norm_grads(tail, 1.0, to_np(mean[-2:]), to_np(rstd[-2:]), tail)
    assert np.all(np.abs(to_np(gg) - dg) <= 1e-5 * (1 + np.abs(dg))) and np.all(np.abs(to_np(gx[-2:]) - dx) <= 2.0 ** -8 * np.abs(dx) + 1e-4)


def test_product_beyond_32_bits():
    m, n, kk = ROWS, COLS, 128
    xq = torch.zeros(m, kk, dtype=E4M3, device="cuda")
    wq = torch.zeros(n, kk, dtype=E4M3, device="cuda")
    xq[-1], wq[-2:] = 2.0, 3.0
    y = torch.empty(m, n, dtype=BF16, device="cuda")
    sbp.sbp_matmul8(one(xq), one(torch.full((m, 1), 0.5, device="cuda")), one(wq), one(torch.full((n // 128, 1), 2.0, device="cuda")), one(y))
    torch.cuda.synchronize()
    assert (y[-1, -2:] == 128 * 6.0).all() and (y[-1, :-2] == 0).all() and not y[:-1].any()
