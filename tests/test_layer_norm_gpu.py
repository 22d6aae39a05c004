"""Layer norm, forward and backward, against the oracle in fp64: every form of the kernels, odd sizes, windows, replicas, empty shards,
rows that are not finite, and the ways the weights' gradients come out.

Tolerances.  u = 2^-24.  A sum of a row is at most 8 elements a thread and chunk one after the other, chunks one after the other and then
a tree of at most 9 + 5 levels: its error is at most D u times the sum of the magnitudes, D = 8 * chunks + 16.  The rest are single roundings,
counted below, and half a step of the result's type."""
import numpy as np
import pytest
import torch
from helpers import make_global, split_cpu, to_np

import paper_2110_15032_b200 as sbp
import sbp_datagen as dg
from oracle import sbp_oracle as O

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
S0, B, P = sbp.S(0), sbp.B, sbp.P_SUM
U = 2.0 ** -24
EPS = 1e-5


def half_step(dtype):
    return 2.0 ** -8 if dtype == BF16 else 2.0 ** -24


def depth(cols):
    chunks = max(4, -(-cols // 4096))                # a chunk of the longest rows is 4096 elements
    return 8 * chunks + 16


def close(got, want, bound, what):
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.size}, worst at {np.argmax(np.abs(got - want) / bound)}: " \
                          f"{np.max(np.abs(got - want) / bound):.2f} of the bound"


def matrix(t, cols):
    return to_np(t).astype(np.float64).reshape(-1, cols)


def check_forward(x, gamma, beta, y, mean, rstd, out_dtype, what=""):
    """One local tensor: host arrays x, gamma, beta (float64 of the stored values) against device results."""
    n = x.shape[1]
    want, m, r = O.layer_norm(x, gamma, beta, EPS)
    d, mag = depth(n), np.abs(x).mean(1)
    dm = (d + 2) * U * mag                                                # the mean's error
    var = 1.0 / r ** 2 - EPS
    dv = (d + 6) * U * var + 2 * dm * np.abs(x - m[:, None]).mean(1) + dm ** 2
    rr = 0.5 * dv * r ** 2 + 4 * U                                        # relative error of rstd
    rr = rr + rr ** 2
    h = np.abs(x - m[:, None]) * r[:, None]
    by = np.abs(gamma) * ((dm * r)[:, None] + h * (rr[:, None] + 4 * U)) + 2 * U * (np.abs(beta) + np.abs(want))
    by = by * (1 + half_step(out_dtype)) + half_step(out_dtype) * np.abs(want) + 1e-38
    close(matrix(y, n), want, by, f"y {what}")
    if mean is not None:
        close(to_np(mean).astype(np.float64).reshape(-1), m, dm + U * np.abs(m) + 1e-40, f"mean {what}")
    if rstd is not None:
        close(to_np(rstd).astype(np.float64).reshape(-1), r, rr * r, f"rstd {what}")


def vectors(cols, seed, dtype=F32):
    return dg.normal(seed, 1, (cols,), 1.0, 0.3, dtype), dg.normal(seed, 2, (cols,), 0.0, 0.5, dtype)


def replicas(t, k):
    return sbp.SbpTensor(tuple(t.shape), t.dtype, B, [t.cuda()] * k)


def run_forward(X, sig, k, out_dtype, gamma, beta, stats=True):
    shape = tuple(X.shape)
    x = make_global(split_cpu(X, sig, k), shape, X.dtype, sig)
    y = sbp.empty_global(shape, out_dtype, sig, k)
    mean = sbp.empty_global(shape[:-1], F32, sig, k) if stats else None
    rstd = sbp.empty_global(shape[:-1], F32, sig, k) if stats else None
    sbp.sbp_layer_norm(x, None if gamma is None else replicas(gamma, k), None if beta is None else replicas(beta, k), y, mean, rstd, EPS)
    torch.cuda.synchronize()
    return x, y, mean, rstd


# every form of the kernels, one element to rows beyond what registers hold; rows fewer than shards
SIZES = [(5, 1), (3, 7), (64, 128), (33, 250), (70, 512), (9, 513), (40, 1024), (17, 1537), (24, 2048), (11, 4096), (7, 4097), (6, 8192),
         (5, 10000), (4, 16384), (3, 16385), (5, 40000), (1, 264), (1300, 256)]


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (F32, F32), (F32, BF16), (BF16, F32)])
def test_forward_forms(rows, cols, dtype, out):
    k = 3
    X = dg.normal(rows * 7 + cols, 0, (rows, cols), 0.7, 2.0, dtype)
    gamma, beta = vectors(cols, cols)
    x, y, mean, rstd = run_forward(X, S0, k, out, gamma, beta)
    for r in range(k):
        check_forward(matrix(x.locals[r], cols), to_np(gamma).astype(np.float64), to_np(beta).astype(np.float64), y.locals[r], mean.locals[r],
                      rstd.locals[r], out, f"shard {r}")


@pytest.mark.parametrize("axis", [0, 1, 2])
def test_axes_and_missing_vectors(axis):
    X = dg.normal(3, axis, (5, 4, 6, 96), 0.0, 1.0, BF16)
    x, y, _, _ = run_forward(X, sbp.S(axis), 4, BF16, None, None, stats=False)
    for r in range(4):
        check_forward(matrix(x.locals[r], 96), np.ones(96), np.zeros(96), y.locals[r], None, None, BF16)


def test_bf16_vectors_and_replicas():
    X = dg.normal(4, 0, (40, 640), 0.0, 1.0, F32)
    gamma, beta = vectors(640, 4, BF16)
    x, y, mean, rstd = run_forward(X, B, 3, F32, gamma, beta)          # three buffers
    for r in range(3):
        check_forward(matrix(x.locals[r], 640), to_np(gamma).astype(np.float64), to_np(beta).astype(np.float64), y.locals[r], mean.locals[r], rstd.locals[r], F32)
    one = sbp.empty_global((40, 640), F32, B, 3, alias_replicas=True)  # and one that all share
    before = sbp.sbp_launch_count()
    sbp.sbp_layer_norm(x, replicas(gamma, 3), replicas(beta, 3), one)
    assert sbp.sbp_launch_count() == before + 1
    torch.cuda.synchronize()
    assert torch.equal(one.locals[0], y.locals[0])


def test_rows_that_are_not_finite_stay_to_themselves():
    X = dg.normal(5, 0, (9, 300), 0.0, 1.0, F32)
    clean = X.clone()
    X[2, 5], X[4, 299], X[7, 0] = float("nan"), float("inf"), float("-inf")
    gamma, beta = vectors(300, 5)
    _, y, _, _ = run_forward(X, S0, 2, F32, gamma, beta)
    _, z, _, _ = run_forward(clean, S0, 2, F32, gamma, beta)
    got, want = torch.cat([t.cpu() for t in y.locals]), torch.cat([t.cpu() for t in z.locals])
    bad = [2, 4, 7]
    assert torch.isnan(got[bad]).all()
    rest = [i for i in range(9) if i not in bad]
    assert torch.equal(got[rest], want[rest])


def test_offset_rows_keep_their_deviation():
    """Rows far from zero: the squares are those of differences, so what is left of the deviation is the type's own."""
    X = dg.normal(6, 0, (12, 2048), 0.0, 1.0, F32) + 3000.0
    gamma, beta = vectors(2048, 6)
    x, y, mean, rstd = run_forward(X, S0, 2, F32, gamma, beta)
    for r in range(2):
        check_forward(matrix(x.locals[r], 2048), to_np(gamma).astype(np.float64), to_np(beta).astype(np.float64), y.locals[r], mean.locals[r], rstd.locals[r], F32)


def windows(rows, cols, k, dtype, skip, pitch_extra):
    """Local tensors that are column blocks of larger buffers, and those buffers."""
    bufs = [torch.full((sbp.sbp_local_shape((rows, cols), S0, k, r)[0], cols + pitch_extra), 7.0, dtype=dtype, device="cuda") for r in range(k)]
    return sbp.SbpTensor((rows, cols), dtype, S0, [b[:, skip:skip + cols] for b in bufs]), bufs


@pytest.mark.parametrize("cols,skip,extra", [(512, 8, 16), (500, 3, 11), (4096, 1, 2)])
def test_windows(cols, skip, extra):
    rows, k = 21, 2
    x, _ = windows(rows, cols, k, BF16, skip, extra)
    for r, t in enumerate(x.locals):
        t.copy_(dg.normal(8, r, tuple(t.shape), 0.0, 1.0, BF16))
    y, bufs = windows(rows, cols, k, F32, skip, extra)
    gamma, beta = vectors(cols, 8)
    sbp.sbp_layer_norm(x, replicas(gamma, k), replicas(beta, k), y)
    torch.cuda.synchronize()
    for r in range(k):
        check_forward(matrix(x.locals[r].contiguous(), cols), to_np(gamma).astype(np.float64), to_np(beta).astype(np.float64), y.locals[r].contiguous(), None, None, F32)
        assert (bufs[r][:, :skip] == 7.0).all() and (bufs[r][:, skip + cols:] == 7.0).all()      # around the window: as it was


def backward(X, DY, k, sig, gsig, gamma, want=(True, True)):
    shape = tuple(X.shape)
    x = make_global(split_cpu(X, sig, k), shape, X.dtype, sig)
    dy = make_global(split_cpu(DY, sig, k), shape, DY.dtype, sig)
    m, r = [], []
    for t in x.locals:
        v = t.double()
        m.append(v.mean(-1).float())
        r.append((v.var(-1, unbiased=False) + EPS).rsqrt().float())
    mean, rstd = sbp.SbpTensor(shape[:-1], F32, sig, m), sbp.SbpTensor(shape[:-1], F32, sig, r)
    dx = sbp.empty_global(shape, X.dtype, sig, k)
    grads = [sbp.empty_global(shape[-1:], F32, gsig, k) if w else None for w in want]
    ws = torch.empty(max(16, sbp.sbp_layer_norm_backward_workspace_bytes(x)), dtype=torch.uint8, device="cuda").fill_(0xFF)
    sbp.sbp_layer_norm_backward(x, None if gamma is None else replicas(gamma, k), mean, rstd, dy, dx, *grads, ws)
    torch.cuda.synchronize()
    return x, dy, mean, rstd, dx, grads


def check_backward(x, dy, mean, rstd, dx, grads, gamma, k, sig, gsig, cols):
    g = np.ones(cols) if gamma is None else to_np(gamma).astype(np.float64)
    sums, mags, rows_all = [], [], 0
    for r in range(1 if sig is B else k):
        X, DY = matrix(x.locals[r], cols), matrix(dy.locals[r], cols)
        M, R = to_np(mean.locals[r]).astype(np.float64).reshape(-1), to_np(rstd.locals[r]).astype(np.float64).reshape(-1)
        want, dgamma, dbeta = O.layer_norm_grads(X, g, M, R, DY)
        h, a, d = np.abs((X - M[:, None]) * R[:, None]), np.abs(DY * g), depth(cols)
        ma, mah = a.mean(1, keepdims=True), (a * h).mean(1, keepdims=True)
        by = R[:, None] * ((d + 10) * U * (ma + h * mah) + 8 * U * (a + ma + h * mah))
        by = by * (1 + half_step(x.dtype)) + half_step(x.dtype) * np.abs(want) + 1e-38
        for q in (range(k) if sig is B else [r]):
            close(matrix(dx.locals[q], cols), want, by, f"grad_x {q}")
        sums.append((dgamma, dbeta))
        mags.append(((np.abs(DY) * h).sum(0), np.abs(DY).sum(0)))
        rows_all += X.shape[0]
    for i, t in enumerate(grads):
        if t is None:
            continue
        # a sum of R terms, in whatever order: at most R additions on a term's way, and three roundings in the term
        whole, mag = sum(s[i] for s in sums), sum(m[i] for m in mags)
        if gsig is P:
            for r in range(k):
                close(to_np(t.locals[r]).astype(np.float64), sums[r][i], (x.locals[r].numel() // cols + 6) * U * mags[r][i] + 1e-38, f"grad {i} of shard {r}")
        elif gsig is B:
            for r in range(k):
                close(to_np(t.locals[r]).astype(np.float64), whole, (rows_all + 6) * U * mag + 1e-38, f"grad {i}, replica {r}")
        else:
            close(np.concatenate([to_np(v) for v in t.locals]).astype(np.float64), whole, (rows_all + 6) * U * mag + 1e-38, f"grad {i}")


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype,dy_dtype", [(BF16, BF16), (F32, F32), (F32, BF16), (BF16, F32)])
def test_backward_forms(rows, cols, dtype, dy_dtype):
    k = 3
    gsig = [P, B, S0][(rows + cols) % 3]
    X, DY = dg.normal(cols, 3, (rows, cols), 0.5, 2.0, dtype), dg.normal(cols, 4, (rows, cols), 0.0, 1.0, dy_dtype)
    gamma, _ = vectors(cols, rows)
    out = backward(X, DY, k, S0, gsig, gamma)
    check_backward(*out, gamma, k, S0, gsig, cols)


@pytest.mark.parametrize("gsig", [P, B, S0])
@pytest.mark.parametrize("rows,cols", [(2, 1000), (300, 96), (50, 20000)])
def test_backward_signatures_and_empty_shards(gsig, rows, cols):
    k = 5                                                        # (2 rows: three shards hold none)
    X, DY = dg.normal(21, 0, (rows, cols), 0.0, 1.0, BF16), dg.normal(21, 1, (rows, cols), 0.0, 1.0, BF16)
    check_backward(*backward(X, DY, k, S0, gsig, None), None, k, S0, gsig, cols)


@pytest.mark.parametrize("gsig", [B, S0])
@pytest.mark.parametrize("cols", [320, 17000])
def test_backward_of_replicas(gsig, cols):
    X, DY = dg.normal(22, 0, (30, cols), 0.0, 1.0, F32), dg.normal(22, 1, (30, cols), 0.0, 1.0, F32)
    gamma, _ = vectors(cols, 22)
    check_backward(*backward(X, DY, 3, B, gsig, gamma), gamma, 3, B, gsig, cols)


@pytest.mark.parametrize("want", [(True, False), (False, True), (False, False)])
def test_backward_without_some_gradients(want):
    X, DY = dg.normal(23, 0, (30, 320), 0.0, 1.0, F32), dg.normal(23, 1, (30, 320), 0.0, 1.0, F32)
    check_backward(*backward(X, DY, 2, S0, P, None, want), None, 2, S0, P, 320)


def test_no_rows_give_zero_gradients():
    x = sbp.empty_global((0, 64), F32, S0, 2)
    st = sbp.empty_global((0,), F32, S0, 2)
    for gsig in (P, B, S0):
        g = sbp.empty_global((64,), F32, gsig, 2)
        sbp.sbp_layer_norm_backward(x, None, st, st, x, x, g, None, torch.empty(16, dtype=torch.uint8, device="cuda"))
        torch.cuda.synchronize()
        assert all((t == 0).all() for t in g.locals)
    sbp.sbp_layer_norm(x, None, None, x, st, st)


def test_gradient_against_differences():
    """The whole chain forward, loss, backward on the device against differences of the fp64 definition."""
    rows, cols, k = 6, 200, 2
    X, W = dg.normal(31, 0, (rows, cols), 0.0, 1.0, F32), dg.normal(31, 1, (rows, cols), 0.0, 1.0, F32)
    gamma, beta = vectors(cols, 31)
    x, dy, mean, rstd, dx, grads = backward(X, W, k, S0, B, gamma)          # the gradient of sum(y W)
    xd, wd, gd, bd = (to_np(t).astype(np.float64) for t in (X, W, gamma, beta))
    loss = lambda x, g: (O.layer_norm(x, g, bd, EPS)[0] * wd).sum()
    got = np.concatenate([to_np(t) for t in dx.locals])
    h = 1e-5
    for i, j in [(0, 0), (3, 99), (5, 199)]:
        e = np.zeros_like(xd)
        e[i, j] = h
        assert abs((loss(xd + e, gd) - loss(xd - e, gd)) / (2 * h) - got[i, j]) < 1e-4
        e = np.zeros(cols)
        e[j] = h
        assert abs((loss(xd, gd + e) - loss(xd, gd - e)) / (2 * h) - to_np(grads[0].locals[0])[j]) < 1e-4


def test_same_bits_every_time_and_in_a_graph():
    rows, cols, k = 700, 1000, 4
    X, DY = dg.normal(41, 0, (rows, cols), 0.0, 1.0, BF16), dg.normal(41, 1, (rows, cols), 0.0, 1.0, BF16)
    x, dy, mean, rstd, dx, grads = backward(X, DY, k, S0, B, None)
    first = [t.clone() for t in dx.locals + grads[0].locals + grads[1].locals]
    ws = torch.empty(sbp.sbp_layer_norm_backward_workspace_bytes(x), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        sbp.sbp_layer_norm_backward(x, None, mean, rstd, dy, dx, *grads, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sbp.sbp_layer_norm_backward(x, None, mean, rstd, dy, dx, *grads, ws)
    for _ in range(3):
        for t in dx.locals + grads[0].locals + grads[1].locals:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, dx.locals + grads[0].locals + grads[1].locals))
