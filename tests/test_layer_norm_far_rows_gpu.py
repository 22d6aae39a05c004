"""Layer norm of rows whose deviation is small beside their mean: equal elements, and elements that differ in their last places.

The mean of n equal fp32 numbers, summed in fp32, is off by some units in the last place; the differences from it are then whole multiples of
such a unit, their sum and the sum of their squares too, so what the mean is off by is found exactly and taken back: y is beta, and where
eps is 0 there is no deviation to divide by and y is NaN.

Tolerance of rows that differ: the first mean is off by at most 30 units, DELTA = 30 * 2^-23 |mean|; what is left of that is the
rounding of a sum of differences of mean magnitude md = mean |x - mean| + DELTA, D u md with D as in the tests of all forms (at most 8
elements a thread and chunk one after the other, a tree above), and of the squares, D u (var + DELTA^2)."""
import numpy as np
import pytest
import torch
from helpers import to_np

import paper_2110_15032_b200 as sbp
import sbp_datagen as dg
from oracle import sbp_oracle as O

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24
# every form: lanes of a warp, a block, two chunks a thread, four, rows that are read again; whole vectors and odd lengths
COLS = [3, 7, 96, 128, 200, 512, 768, 1000, 1537, 2048, 4096, 4099, 5000, 8192, 16384, 16381, 16392, 40000, 40001, 300000]


def one(t):
    return sbp.SbpTensor(tuple(t.shape), t.dtype, sbp.B, [t])


def run(x, beta, eps, out=F32, gamma=None):
    rows, cols = x.shape
    y, mean, rstd = (sbp.empty_global(s, d, sbp.B, 1) for s, d in (((rows, cols), out), ((rows,), F32), ((rows,), F32)))
    sbp.sbp_layer_norm(one(x), None if gamma is None else one(gamma), one(beta), y, mean, rstd, eps)
    torch.cuda.synchronize()
    return y.locals[0], mean.locals[0], rstd.locals[0]


@pytest.mark.parametrize("cols", COLS)
def test_rows_of_equal_elements_give_beta(cols):
    values = [0.1, 1.1, -0.7, 12345.678, 3000.3, -7.3e-5, 1e-30, 33333.332, 0.0] + ([1e30] if cols <= 4096 else [])
    v = torch.tensor(values, dtype=F32, device="cuda")
    x = v[:, None].expand(-1, cols).contiguous()
    beta = dg.normal(cols, 0, (cols,), 0.0, 1.0, F32).cuda()
    gamma = dg.normal(cols, 1, (cols,), 1.0, 0.3, F32).cuda()
    for out in (F32, BF16):
        y, mean, rstd = run(x, beta, 1e-5, out, gamma)
        assert torch.equal(y, beta.to(out).expand_as(y)), [i for i in range(len(values)) if not torch.equal(y[i], beta.to(out))]
        assert torch.equal(mean, v)
        small = v.abs() < 1e20                       # (1e30: the first mean's differences, squared, leave fp32)
        assert torch.allclose(rstd[small], torch.full_like(v, 1e-5).rsqrt()[small], rtol=4 * U, atol=0)
    y, mean, rstd = run(x[small], beta, 0.0)
    assert torch.isnan(y).all() and torch.equal(mean, v[small]) and torch.isinf(rstd).all()


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("base", [1.1, 12345.678, -3000.3])
def test_rows_that_differ_in_their_last_places(cols, base):
    g = torch.Generator().manual_seed(cols)
    step = float(np.spacing(np.float32(abs(base))))
    x = (torch.tensor(base, dtype=F32) + step * torch.randint(-9, 10, (6, cols), generator=g).float()).cuda()
    gamma, beta = dg.normal(cols, 2, (cols,), 1.0, 0.3, F32).cuda(), dg.normal(cols, 3, (cols,), 0.0, 1.0, F32).cuda()
    X, G, Bt = (to_np(t).astype(np.float64) for t in (x, gamma, beta))
    for eps in (1e-5, 1e-12):
        e = float(np.float32(eps))
        y, mean, rstd = run(x, beta, eps, F32, gamma)
        want, m, r = O.layer_norm(X, G, Bt, e)
        d = 8 * max(4, -(-cols // 4096)) + 16
        delta = 30 * 2.0 ** -23 * np.abs(m)
        dev, var = np.abs(X - m[:, None]), 1 / r ** 2 - e
        dm = (d + 4) * U * (dev.mean(1) + delta)
        dv = (d + 6) * U * (var + delta ** 2) + 2 * dm * dev.mean(1) + dm ** 2
        rr = 0.5 * dv * r ** 2
        assert np.all(rr < 0.1)
        rr = rr * 1.2 + 4 * U                        # (1 + t)^(-1/2) beyond its first order, t up to 0.2
        by = np.abs(G) * ((dm * r)[:, None] * (1 + rr[:, None]) + dev * r[:, None] * (rr[:, None] + 4 * U)) + 2 * U * (np.abs(Bt) + np.abs(want))
        got = to_np(y).astype(np.float64)
        assert np.all(np.abs(got - want) <= by), f"eps {eps}: {np.max(np.abs(got - want) / by)} of the bound, {np.max(np.abs(got - want))}"
        assert np.all(np.abs(to_np(mean) - m) <= dm + U * np.abs(m)) and np.all(np.abs(to_np(rstd) - r) <= rr * r)
