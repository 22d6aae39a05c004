"""Windows into larger buffers where layer norm and the 8-bit entry points take them: the gradients of layer norm (rows in registers, in odd pieces, read
again from L2), both GeLU passes, and results of the 8-bit product in every signature and kind of form.  What lies around a window that is
read is NaN, what lies around one that is written stays as it was."""
import numpy as np
import pytest
import torch
from helpers import make_global, split_cpu, to_np
from test_blocks8_gpu import close, gelu_bound, half_step, np8, same_blocks
from test_layer_norm_gpu import EPS, check_backward, check_forward, matrix, replicas, vectors
from test_matmul8_gpu import ROWS, Operand, expected

import paper_2110_15032_b200 as sbp
import sbp_datagen as dg
from oracle import sbp_oracle as O

pytestmark = pytest.mark.gpu
F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
S0, S1, B, P = sbp.S(0), sbp.S(1), sbp.B, sbp.P_SUM
U = 2.0 ** -24


class Windows:
    """Local tensors as column blocks of larger buffers, and those buffers."""

    def __init__(self, shape, dtype, sig, k, skip, extra, around=float("nan")):
        self.cols, self.skip, self.bufs, locs = [], skip, [], []
        for r in range(k):
            shp = sbp.sbp_local_shape(shape, sig, k, r, dtype)
            buf = torch.full((*shp[:-1], shp[-1] + extra), around, dtype=F32, device="cuda").to(dtype)
            self.bufs.append(buf)
            self.cols.append(shp[-1])
            locs.append(buf[..., skip:skip + shp[-1]])
        self.t = sbp.SbpTensor(shape, dtype, sig, locs)
        self.around = around

    def fill(self, parts):
        for t, v in zip(self.t.locals, parts):
            t.copy_(v)
        return self

    def dense(self):
        return sbp.SbpTensor(self.t.shape, self.t.dtype, self.t.sig, [t.contiguous() for t in self.t.locals])

    def untouched(self):
        for b, c in zip(self.bufs, self.cols):
            b = b.float()
            assert (b[..., :self.skip] == self.around).all() and (b[..., self.skip + c:] == self.around).all()


PADS = [(8, 16), (3, 7)]       # whole vectors still, and not


@pytest.mark.parametrize("skip,extra", PADS)
@pytest.mark.parametrize("cols", [96, 500, 1024, 4096, 4097, 8200, 20000])
@pytest.mark.parametrize("gsig", [P, B, S0])
@pytest.mark.parametrize("dtype,dy_dtype", [(BF16, BF16), (F32, BF16)])
def test_windows_of_layer_norm_gradients(skip, extra, cols, gsig, dtype, dy_dtype):
    rows, k = 23, 3
    gamma, beta = vectors(cols, 9)
    x = Windows((rows, cols), dtype, S0, k, skip, extra).fill(split_cpu(dg.normal(cols, 0, (rows, cols), 0.5, 2.0, dtype), S0, k))
    dy = Windows((rows, cols), dy_dtype, S0, k, skip, extra).fill(split_cpu(dg.normal(cols, 1, (rows, cols), 0.0, 1.0, dy_dtype), S0, k))
    dx = Windows((rows, cols), dtype, S0, k, skip, extra, 7.0)
    y = Windows((rows, cols), dy_dtype, S0, k, skip, extra, 7.0)
    mean, rstd = sbp.empty_global((rows,), F32, S0, k), sbp.empty_global((rows,), F32, S0, k)
    sbp.sbp_layer_norm(x.t, replicas(gamma, k), replicas(beta, k), y.t, mean, rstd, EPS)
    grads = [sbp.empty_global((cols,), F32, gsig, k) for _ in range(2)]
    ws = torch.empty(max(16, sbp.sbp_layer_norm_backward_workspace_bytes(x.t)), dtype=torch.uint8, device="cuda").fill_(0xFF)
    sbp.sbp_layer_norm_backward(x.t, replicas(gamma, k), mean, rstd, dy.t, dx.t, *grads, ws)
    torch.cuda.synchronize()
    g, b = to_np(gamma).astype(np.float64), to_np(beta).astype(np.float64)
    for r in range(k):
        check_forward(matrix(x.dense().locals[r], cols), g, b, y.dense().locals[r], mean.locals[r], rstd.locals[r], dy_dtype, f"shard {r}")
    check_backward(x.dense(), dy.dense(), mean, rstd, dx.dense(), grads, gamma, k, S0, gsig, cols)
    dx.untouched()
    y.untouched()


@pytest.mark.parametrize("skip,extra", [(16, 32), (3, 7)])
@pytest.mark.parametrize("shape,sig", [((40, 544), S0), ((40, 544), S1), ((3, 7, 400), sbp.S(1)), ((21, 1003), S0)])
@pytest.mark.parametrize("zt,yt", [(BF16, BF16), (F32, F32), (BF16, F32), (F32, BF16)])
def test_windows_of_gelu_and_its_gradient(skip, extra, shape, sig, zt, yt):
    k = 2
    z = Windows(shape, zt, sig, k, skip, extra).fill(split_cpu(dg.normal(5, 0, shape, 0.0, 2.0, zt), sig, k))
    dy = Windows(shape, yt, sig, k, skip, extra).fill(split_cpu(dg.normal(5, 1, shape, 0.0, 1.0, yt), sig, k))
    y, dz = Windows(shape, yt, sig, k, skip, extra, 7.0), Windows(shape, zt, sig, k, skip, extra, 7.0)
    q = Windows(shape, E4M3, sig, k, skip, extra, 7.0)
    s = sbp.empty_global(sbp.sbp_scales_shape(shape, sig, k), F32, sig, k)
    sbp.sbp_gelu_save8(z.t, y.t, q.t, s)
    sbp.sbp_gelu_save8_backward(q.t, s, dy.t, dz.t)
    torch.cuda.synchronize()
    for r in range(k):
        cols = z.cols[r]
        v, d, sc = matrix(z.dense().locals[r], cols), matrix(dy.dense().locals[r], cols), to_np(s.locals[r])
        same_blocks(v, q.dense().locals[r], s.locals[r], 0, f"shard {r}")
        want = O.gelu_from_erfc(v)
        close(matrix(y.dense().locals[r], cols), want, gelu_bound(v, want, yt), "y")
        v = O.dequantize8(np8(q.dense().locals[r]).reshape(v.shape), sc.reshape(v.shape[0], -1))
        want = d * O.gelu_slope(v)
        # each of the slope's two terms to 2^-20 and what its exponent's rounding brings, and half a step of the result
        terms = 0.5 * O._erfc(-v / np.sqrt(2)) + np.abs(v) * np.exp(-0.5 * v * v) / np.sqrt(2 * np.pi)
        by = np.abs(d) * (terms * (2.0 ** -20 + 2 * v * v * U) + 0.8 * np.abs(v) * U)
        close(matrix(dz.dense().locals[r], cols), want, by * (1 + half_step(zt)) + half_step(zt) * np.abs(want) + 2.0 ** -126, "grad_z")
    for t in (y, dz, q):
        t.untouched()


# the library's choice for few rows, the pair form, and single tiles whose contraction is shared, exchanged and not
@pytest.mark.parametrize("m,n,form", [(9, 700, None), (140, 270, None), (1100, 1350, (256, 1, False)), (140, 270, (128, 4, False)), (140, 270, (32, 4, True)),
                                      (140, 270, (64, 1, True))])
@pytest.mark.parametrize("sig", ["rows", "columns", "partial", "fused_b", "fused_s0", "fused_s1", "whole"])
def test_windows_of_results_of_products(m, n, form, sig):
    rng = np.random.default_rng(m + n)
    sx, sw, sy = ROWS[sig]
    k, kk = 2, 2 * 1040
    x, w = Operand(m, kk, sx, k, False, rng, True), Operand(n, kk, sw, k, True, rng, True)
    want = expected(x, w, sig, k, m, n)
    try:
        if form:
            sbp.sbp_matmul8_set_form(*form)
        for dtype, skip, extra in ((F32, 4, 8), (F32, 3, 9), (BF16, 8, 16), (BF16, 5, 7), (BF16, 4, 4)):
            y = Windows((m, n), dtype, sy, k, skip, extra, 7.0)
            sbp.sbp_matmul8(x.values, x.scales, w.values, w.scales, y.t)
            torch.cuda.synchronize()
            for r in range(k):
                assert np.array_equal(to_np(y.dense().locals[r]), to_np(torch.from_numpy(want[r][0]).float().to(dtype))), (dtype, skip, r)
            y.untouched()
    finally:
        sbp.sbp_matmul8_set_form()
