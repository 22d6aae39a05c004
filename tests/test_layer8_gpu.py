"""One transformer MLP layer trained in 8 bits, as a program makes the calls, weights split over the devices (the paper's Megatron-style
signatures): layer norm, quantisation, product, GeLU with checkpoint, quantisation, product whose partial results are summed; and back to the
gradients of the input, of both weights and of gamma and beta.  Every step is held to the fp64 definition of what it was given, and the
gradients to those of the same layer without quantisation.

Quantising moves an element by at most 2^-4 of itself (half a step of e4m3), or half its smallest step, 2^-10 scale <= 2^-10 * 2^-8 * 2 max / 1.75,
so |q(x) - x| <= 2^-4 |x| + 2^-17 max|x|; the bounds below carry that through the products, element by element."""
import numpy as np
import pytest
import torch
from helpers import split_cpu, to_np

import paper_2110_15032_b200 as sbp
import sbp_datagen as dg
from oracle import sbp_oracle as O

pytestmark = pytest.mark.gpu
F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
S0, S1, B, P = sbp.S(0), sbp.S(1), sbp.B, sbp.P_SUM
TILES, TRANS = sbp.SBP_QUANT_TILES, sbp.SBP_TRANS_X
EPS = 1e-5


def whole(t):
    """The global tensor in fp64."""
    loc = [to_np(v).astype(np.float64) for v in t.locals]
    sig = t.sig
    return loc[0] if sig == B else np.concatenate(loc, sig.axis) if sig.kind == 0 else sum(loc)


class Blocks:
    """x in 8 bits."""

    def __init__(self, x, flags=0):
        shape, sig = (x.shape[::-1], x.sig if x.sig == B else sbp.S(1 - x.sig.axis)) if flags & TRANS else (x.shape, x.sig)
        self.tiles = bool(flags & TILES)
        alias = sig == B
        self.values = sbp.empty_global(shape, E4M3, sig, x.k, alias_replicas=alias)
        self.scales = sbp.empty_global(sbp.sbp_scales_shape(shape, sig, x.k, flags & TILES), F32, sig, x.k, alias_replicas=alias)
        sbp.sbp_quantize8(x, self.values, self.scales, flags)

    def whole(self):
        """What it stands for, in fp64."""
        loc = [O.dequantize8(v.float().cpu().numpy(), to_np(s), self.tiles) for v, s in zip(self.values.locals, self.scales.locals)]
        sig = self.values.sig
        return loc[0] if sig == B else np.concatenate(loc, sig.axis)


def product(x, w, shape, dtype, sig):
    y = sbp.empty_global(shape, dtype, sig, x.values.k, alias_replicas=sig == B)
    sbp.sbp_matmul8(x.values, x.scales, w.values, w.scales, y)
    return y


def check(got, want, mag, dtype, kk, what):
    half = 2.0 ** -8 if dtype is BF16 else 2.0 ** -24
    by = (128 * 2.0 ** -23 + (kk / 128 + 12) * 2.0 ** -24) * mag
    by = by * (1 + half) + half * np.abs(want) + 1e-38
    assert np.all(np.abs(got - want) <= by), f"{what}: {np.max(np.abs(got - want) / by)} of the bound"


def check_product(y, a, b, dtype, what):
    check(whole(y), a @ b.T, np.abs(a) @ np.abs(b).T, dtype, a.shape[1], what)


def off(x):
    """How far quantising may move the elements of x."""
    return 2.0 ** -4 * np.abs(x) + 2.0 ** -17 * np.abs(x).max()


@pytest.mark.parametrize("m,h,f,k", [(192, 256, 1024, 4), (300, 400, 1040, 2), (1, 128, 256, 2)])
def test_forward_and_backward(m, h, f, k):
    X = dg.normal(50, 0, (m, h), 0.3, 1.5, BF16)
    W1, W2 = dg.normal(50, 1, (h, f), 0.0, h ** -0.5, BF16), dg.normal(50, 2, (f, h), 0.0, f ** -0.5, BF16)
    gamma, beta = dg.normal(50, 3, (h,), 1.0, 0.2, F32), dg.normal(50, 4, (h,), 0.0, 0.2, F32)
    DY = dg.normal(50, 5, (m, h), 0.0, 1.0, BF16)
    one = lambda t: sbp.SbpTensor(tuple(t.shape), t.dtype, B, [t.cuda()] * k)
    cut = lambda t, sig: sbp.SbpTensor(tuple(t.shape), t.dtype, sig, [v.cuda() for v in split_cpu(t, sig, k)])
    room = lambda shape, dtype, sig: sbp.empty_global(shape, dtype, sig, k, alias_replicas=sig == B)

    # weights in 8 bits, for the products of the forward pass ([N, K]) and for those of the input's gradients
    w1, w2 = cut(W1, S1), cut(W2, S0)
    w1f, w1b = Blocks(w1, TILES | TRANS), Blocks(w1, TILES)
    w2f, w2b = Blocks(w2, TILES | TRANS), Blocks(w2, TILES)
    assert np.array_equal(w1f.whole().T, w1b.whole()) or h % 128 or (f // k) % 128      # the same tiles, either way round

    # forward
    x, g, b = one(X), one(gamma), one(beta)
    n, mean, rstd = room((m, h), BF16, B), room((m,), F32, B), room((m,), F32, B)
    sbp.sbp_layer_norm(x, g, b, n, mean, rstd, EPS)
    n8 = Blocks(n)
    z = product(n8, w1f, (m, f), BF16, S1)
    a, z8v = room((m, f), BF16, S1), room((m, f), E4M3, S1)
    z8s = room(sbp.sbp_scales_shape((m, f), S1, k), F32, S1)
    sbp.sbp_gelu_save8(z, a, z8v, z8s)
    a8 = Blocks(a)
    y = product(a8, w2f, (m, h), BF16, B)

    # backward
    dy = one(DY)
    dy8, dy8t = Blocks(dy), Blocks(dy, TRANS)
    a8t = Blocks(a, TRANS)
    dw2 = product(a8t, dy8t, (f, h), F32, S0)                     # A^T dY
    da = product(dy8, w2b, (m, f), BF16, S1)                      # dY W2^T
    dz = room((m, f), BF16, S1)
    sbp.sbp_gelu_save8_backward(z8v, z8s, da, dz)
    dz8, dz8t = Blocks(dz), Blocks(dz, TRANS)
    n8t = Blocks(n, TRANS)
    dw1 = product(n8t, dz8t, (h, f), F32, S1)                     # N^T dZ
    dn = product(dz8, w1b, (m, h), F32, B)                        # dZ W1^T, summed over the devices
    dx, dg_, db_ = room((m, h), BF16, B), room((h,), F32, B), room((h,), F32, B)
    ws = torch.empty(max(16, sbp.sbp_layer_norm_backward_workspace_bytes(x)), dtype=torch.uint8, device="cuda")
    sbp.sbp_layer_norm_backward(x, g, mean, rstd, dn, dx, dg_, db_, ws)
    torch.cuda.synchronize()

    # every product from what it was given
    check_product(z, n8.whole(), w1f.whole(), BF16, "z")
    check_product(y, a8.whole(), w2f.whole(), BF16, "y")
    check_product(dw2, a8t.whole(), dy8t.whole(), F32, "dW2")
    check_product(da, dy8.whole(), w2b.whole(), BF16, "dA")
    check_product(dw1, n8t.whole(), dz8t.whole(), F32, "dW1")
    check_product(dn, dz8.whole(), w1b.whole(), F32, "dN")
    # every quantised tensor from what it was made of
    for q, t, name in ((n8, n, "n"), (a8, a, "a"), (dy8, dy, "dy"), (dz8, dz, "dz"), (w1b, w1, "w1"), (w2b, w2, "w2")):
        assert np.all(np.abs(q.whole() - whole(t)) <= off(whole(t))), name
    for q, t, name in ((n8t, n, "n"), (a8t, a, "a"), (dz8t, dz, "dz"), (w1f, w1, "w1"), (w2f, w2, "w2")):
        assert np.all(np.abs(q.whole().T - whole(t)) <= off(whole(t))), name
    # the gradient of the layer, from the gradient that the products brought
    wx, wg, wb = O.layer_norm_grads(whole(x), to_np(gamma).astype(np.float64), whole(mean), whole(rstd), whole(dn))
    scale = np.abs(whole(rstd))[:, None] * (np.abs(whole(dn)) @ np.ones((h, 1)) / h + np.abs(whole(dn))) * 8 + 1e-30
    assert np.all(np.abs(whole(dx) - wx) <= 2.0 ** -8 * np.abs(wx) + 2.0 ** -15 * scale)

    # gradients of the weights against the layer in fp64, without quantisation, element by element
    N, A, DYd, DZ = whole(n), whole(a), whole(dy), whole(dz)
    for got, p, q, name in ((dw2, A, DYd, "dW2"), (dw1, N, DZ, "dW1")):
        exact = p.T @ q
        by = off(p).T @ np.abs(q) + np.abs(p).T @ off(q) + off(p).T @ off(q) + 2e-5 * (np.abs(p).T @ np.abs(q))
        assert np.all(np.abs(whole(got) - exact) <= by), name
