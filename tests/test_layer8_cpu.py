"""Layer norm, 8-bit blocks and 8-bit products without a GPU: what the entry points refuse, the shape of scales, and the oracle's
definitions against hand values, the bit patterns of e4m3 and finite differences."""
import numpy as np
import pytest
import torch

import paper_2110_15032_b200 as sbp
from oracle import sbp_oracle as O

F32, BF16, I64, E4M3 = torch.float32, torch.bfloat16, torch.int64, torch.float8_e4m3fn
S0, S1, B, P = sbp.S(0), sbp.S(1), sbp.B, sbp.P_SUM


class Stream:
    cuda_stream = 0


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2110_15032_b200.build import build
    build()


def host(shape, dtype, sig, k, pshape=None):
    n = k if pshape is None else pshape[0] * pshape[1]
    return sbp.SbpTensor(shape, dtype, sig, [torch.zeros(sbp.sbp_local_shape(shape, sig, pshape or k, r, dtype), dtype=dtype) for r in range(n)], pshape)


def status(fn, *a, **kw):
    try:
        fn(*a, stream=Stream(), **kw)
    except sbp.SbpError as e:
        return e.name[4:]
    return "OK"


def window(t):
    """The same global tensor in rows of a larger buffer."""
    locs = []
    for v in t.locals:
        buf = torch.zeros((*v.shape[:-1], v.shape[-1] + 16), dtype=v.dtype)
        locs.append(buf[..., :v.shape[-1]])
    return sbp.SbpTensor(t.shape, t.dtype, t.sig, locs)


def test_layer_norm_refusals():
    def forward(x=None, gamma="ok", beta="ok", y=None, mean="ok", rstd="ok", eps=1e-5):
        x = x or host((6, 10), F32, S0, 2)
        vec = lambda t: host((10,), F32, B, 2) if t == "ok" else t
        stat = lambda t: host((6,), F32, S0, 2) if t == "ok" else t
        return status(sbp.sbp_layer_norm, x, vec(gamma), vec(beta), y or host((6, 10), BF16, S0, 2), stat(mean), stat(rstd), eps)

    assert forward(x=host((6, 10), F32, S1, 2)) == "ERR_UNSUPPORTED"          # split along the rows themselves
    assert forward(x=host((6, 10), F32, P, 2)) == "ERR_SIGNATURE"
    assert forward(x=host((6, 10), I64, S0, 2)) == "ERR_DTYPE"
    assert forward(x=host((6, 10), E4M3, S0, 2)) == "ERR_DTYPE"
    assert forward(x=host((10,), F32, S0, 2)) == "ERR_SHAPE"
    assert forward(x=host((6, 0), F32, S0, 2), y=host((6, 0), F32, S0, 2)) == "ERR_SHAPE"
    assert forward(x=host((6, 10), F32, (S0, S0), 4, (2, 2))) == "ERR_UNSUPPORTED"
    assert forward(y=host((6, 11), F32, S0, 2)) == "ERR_SHAPE"
    assert forward(y=host((6, 10), F32, B, 2)) == "ERR_SIGNATURE"
    assert forward(y=host((6, 10), F32, S0, 3)) == "ERR_INVALID_ARG"
    assert forward(y=host((6, 10), I64, S0, 2)) == "ERR_DTYPE"
    assert forward(gamma=host((9,), F32, B, 2)) == "ERR_SHAPE"
    assert forward(gamma=host((10,), F32, S0, 2)) == "ERR_SIGNATURE"
    assert forward(beta=host((10,), I64, B, 2)) == "ERR_DTYPE"
    assert forward(mean=host((6,), BF16, S0, 2)) == "ERR_DTYPE"
    assert forward(rstd=host((6,), F32, B, 2)) == "ERR_SIGNATURE"
    assert forward(rstd=host((6, 1), F32, S0, 2)) == "ERR_SHAPE"
    for eps in (-1e-5, float("nan"), float("inf")):
        assert forward(eps=eps) == "ERR_INVALID_ARG"


def test_layer_norm_backward_refusals():
    ws = torch.zeros(1 << 20, dtype=torch.uint8)

    def backward(x=None, gy=None, gx=None, mean=None, gg="ok", gb="ok", ws=ws):
        vec = lambda t: host((10,), F32, P, 2) if t == "ok" else t
        st = lambda: host((6,), F32, S0, 2)
        return status(sbp.sbp_layer_norm_backward, x or host((6, 10), F32, S0, 2), host((10,), F32, B, 2), mean or st(), st(),
                      gy or host((6, 10), F32, S0, 2), gx or host((6, 10), F32, S0, 2), vec(gg), vec(gb), ws)

    assert backward(gx=host((6, 10), BF16, S0, 2)) == "ERR_DTYPE"              # grad_x is as x
    assert backward(gy=host((5, 10), F32, S0, 2)) == "ERR_SHAPE"
    assert backward(mean=host((6,), F32, B, 2)) == "ERR_SIGNATURE"
    assert backward(gg=host((10,), F32, B, 2)) == "ERR_SIGNATURE"              # the two gradients differ
    assert backward(gg=host((10,), BF16, P, 2)) == "ERR_DTYPE"
    assert backward(gb=host((10,), F32, sbp.P_MAX, 2)) == "ERR_SIGNATURE"
    assert backward(gb=host((11,), F32, P, 2)) == "ERR_SHAPE"
    assert backward(ws=None) == "ERR_WORKSPACE"
    assert backward(ws=torch.zeros(8, dtype=torch.uint8)) == "ERR_WORKSPACE"
    assert backward(ws=ws[1:]) == "ERR_ALIGNMENT"
    xb = host((6, 10), F32, B, 2)
    stb = host((6,), F32, B, 2)
    assert status(sbp.sbp_layer_norm_backward, xb, None, stb, stb, xb, xb, host((10,), F32, P, 2), None, ws) == "ERR_SIGNATURE"
    assert sbp.sbp_layer_norm_backward_workspace_bytes(host((6, 10), F32, S1, 2)) == 0
    assert sbp.sbp_layer_norm_backward_workspace_bytes(host((6, 10), F32, S0, 2)) >= 2 * 2 * 10 * 4


def test_blocks_refusals():
    x, q, s = host((6, 300), F32, S0, 2), host((6, 300), E4M3, S0, 2), host((6, 3), F32, S0, 2)
    quant = lambda *a, **kw: status(sbp.sbp_quantize8, *a, **kw)
    assert quant(x, host((6, 300), BF16, S0, 2), s) == "ERR_DTYPE"
    assert quant(host((6, 300), I64, S0, 2), q, s) == "ERR_DTYPE"
    assert quant(host((6, 300), E4M3, S0, 2), q, s) == "ERR_DTYPE"
    assert quant(host((6, 300), F32, P, 2), host((6, 300), E4M3, P, 2), host((6, 3), F32, P, 2)) == "ERR_SIGNATURE"
    assert quant(x, q, host((6, 2), F32, S0, 2)) == "ERR_SHAPE"
    assert quant(x, q, host((5, 3), F32, S0, 2)) == "ERR_SHAPE"
    assert quant(x, q, host((6, 3), BF16, S0, 2)) == "ERR_DTYPE"
    assert quant(x, q, host((6, 3), F32, B, 2)) == "ERR_SIGNATURE"
    assert quant(x, q, window(s)) == "ERR_UNSUPPORTED"
    assert quant(x, host((6, 301), E4M3, S0, 2), s) == "ERR_SHAPE"
    assert quant(x, host((6, 300), E4M3, B, 2), host((6, 3), F32, B, 2)) == "ERR_SIGNATURE"
    assert quant(x, host((6, 300), E4M3, S0, 3), host((6, 3), F32, S0, 3)) == "ERR_INVALID_ARG"
    assert quant(x, q, s, flags=1) == "ERR_INVALID_ARG"
    assert quant(x, q, s, flags=sbp.SBP_QUANT_TILES) == "ERR_SHAPE"            # tiles want [2, 3] scales
    assert quant(x, q, s, flags=sbp.SBP_TRANS_X) == "ERR_SHAPE"
    assert quant(x, host((300, 6), E4M3, S0, 2), host((300, 1), F32, S0, 2), flags=sbp.SBP_TRANS_X) == "ERR_SIGNATURE"
    x3 = host((2, 3, 8), F32, S0, 2)
    assert quant(x3, host((2, 3, 8), E4M3, S0, 2), host((2, 3, 1), F32, S0, 2), flags=sbp.SBP_TRANS_X) == "ERR_SHAPE"
    gelu = lambda *a: status(sbp.sbp_gelu_save8, *a)
    assert gelu(x, host((6, 301), F32, S0, 2), q, s) == "ERR_SHAPE"
    assert gelu(x, host((6, 300), I64, S0, 2), q, s) == "ERR_DTYPE"
    assert gelu(host((6, 300), F32, P, 2), host((6, 300), F32, P, 2), q, s) == "ERR_SIGNATURE"
    back = lambda *a: status(sbp.sbp_gelu_save8_backward, *a)
    assert back(q, s, x, host((6, 300), F32, S1, 2)) == "ERR_SIGNATURE"
    assert back(q, host((1 * 2, 3), F32, S0, 2), x, x) == "ERR_SHAPE"          # a scale a tile
    assert back(host((6, 300), E4M3, P, 2), host((6, 3), F32, P, 2), x, x) == "ERR_SIGNATURE"


def test_matmul8_refusals():
    x, xs = host((6, 300), E4M3, B, 2), host((6, 3), F32, B, 2)
    w, ws, y = host((10, 300), E4M3, S0, 2), host((2, 3), F32, S0, 2), host((6, 10), F32, S1, 2)
    mul = lambda *a: status(sbp.sbp_matmul8, *a)
    assert mul(host((6, 300), F32, B, 2), xs, w, ws, y) == "ERR_DTYPE"
    assert mul(x, xs, host((10, 299), E4M3, S0, 2), ws, y) == "ERR_SHAPE"
    assert mul(x, host((6, 2), F32, B, 2), w, ws, y) == "ERR_SHAPE"
    assert mul(x, xs, w, host((3, 3), F32, S0, 2), y) == "ERR_SHAPE"
    assert mul(x, xs, w, ws, host((6, 10), E4M3, S1, 2)) == "ERR_DTYPE"
    assert mul(x, xs, w, ws, host((6, 10), F32, S0, 2)) == "ERR_SIGNATURE"
    assert mul(host((6, 300), E4M3, S0, 2), host((6, 3), F32, S0, 2), w, ws, y) == "ERR_SIGNATURE"     # not a row of Table 1
    assert mul(x, window(xs), w, ws, y) == "ERR_UNSUPPORTED"
    assert mul(x, host((6, 3), F32, S0, 2), w, ws, y) == "ERR_SIGNATURE"
    assert mul(host((6, 300), E4M3, (B, B), 4, (2, 2)), xs, w, ws, y) == "ERR_UNSUPPORTED"


def test_other_entry_points_refuse_8_bit_values():
    q = host((8, 16), E4M3, S0, 2)
    assert status(sbp.sbp_boxing, q, host((8, 16), E4M3, B, 2)) == "ERR_DTYPE"
    assert status(sbp.sbp_boxing_shard, q, host((8, 16), E4M3, B, 2), 0) == "ERR_DTYPE"
    assert status(sbp.sbp_matmul, q, host((16, 8), E4M3, B, 2), host((8, 8), F32, S0, 2)) == "ERR_DTYPE"
    with pytest.raises(sbp.SbpError):
        sbp.sbp_view_b_to_s(host((8, 16), E4M3, B, 2), 0)
    assert sbp.sbp_boxing_host_workspace_bytes(q, host((8, 16), E4M3, B, 2)) == 0


@pytest.mark.parametrize("shape", [(6, 300), (1, 1), (1000, 129), (385, 385), (3, 4, 500), (257,), (0, 256), (130, 0)])
@pytest.mark.parametrize("k", [1, 2, 3, 8, 16])
def test_every_shard_gets_the_scales_of_its_own_blocks(shape, k):
    up = lambda n: -(-n // 128)
    for sig in [sbp.S(i) for i in range(len(shape))] + [B]:
        for flags in (0, sbp.SBP_QUANT_TILES) if len(shape) == 2 else (0,):
            scales = sbp.sbp_scales_shape(shape, sig, k, flags)
            for r in range(k):
                v, s = sbp.sbp_local_shape(shape, sig, k, r, E4M3), sbp.sbp_local_shape(scales, sig, k, r)
                want = list(v)
                want[-1] = up(v[-1])
                if flags:
                    want[0] = up(v[0])
                assert s == tuple(want), (sig, flags, r)


def test_e4m3_rounding_is_that_of_the_bit_patterns():
    """Every e4m3 number stands still; halfway between neighbours the even one is taken."""
    codes = torch.arange(0, 127, dtype=torch.uint8)
    v = codes.view(E4M3).double().numpy()
    assert v[-1] == 448.0 and np.all(np.diff(v) > 0)
    assert np.array_equal(O.round_to_e4m3(v), v) and np.array_equal(O.round_to_e4m3(-v), -v)
    mid = (v[:-1] + v[1:]) / 2
    even = np.where(np.arange(126) % 2 == 0, v[:-1], v[1:])
    assert np.array_equal(O.round_to_e4m3(mid), even)
    assert np.array_equal(O.round_to_e4m3(mid * (1 - 1e-12)), v[:-1]) and np.array_equal(O.round_to_e4m3(mid * (1 + 1e-12)), v[1:])
    assert np.isnan(O.round_to_e4m3([np.inf, -np.inf, np.nan])).all()


def test_quantize8_by_hand():
    x = np.zeros((2, 130))
    x[0, 0], x[0, 1], x[0, 129] = 448.0, -1.0, 449.0
    x[1, 0], x[1, 129] = np.inf, 2.0 ** -140
    q, s = O.quantize8(x)
    assert s.tolist() == [[1.0, 2.0], [1.0, 2.0 ** -126]]
    assert q[0, 0] == 448.0 and q[0, 1] == -1.0 and q[0, 129] == 224.0 and np.isnan(q[1, 0]) and q[1, 129] == 0.0
    q, s = O.quantize8(x, tiles=True)
    assert s.tolist() == [[1.0, 2.0]]
    assert np.array_equal(O.dequantize8(q, s, True)[0, [0, 1, 129]], [448.0, -1.0, 448.0])


def test_oracle_gradients_against_differences():
    rng = np.random.default_rng(7)
    x, gamma, beta, dy = rng.normal(1, 2, (5, 13)), rng.normal(1, 0.3, 13), rng.normal(0, 1, 13), rng.normal(0, 1, (5, 13))
    _, mean, rstd = O.layer_norm(x, gamma, beta, 1e-5)
    dx, dg, db = O.layer_norm_grads(x, gamma, mean, rstd, dy)
    loss = lambda x, g, b: float((O.layer_norm(x, g, b, 1e-5)[0] * dy).sum())
    h = 1e-6
    for i, j in [(0, 0), (2, 7), (4, 12)]:
        e = np.zeros_like(x)
        e[i, j] = h
        assert abs((loss(x + e, gamma, beta) - loss(x - e, gamma, beta)) / (2 * h) - dx[i, j]) < 1e-7
        e = np.zeros(13)
        e[j] = h
        assert abs((loss(x, gamma + e, beta) - loss(x, gamma - e, beta)) / (2 * h) - dg[j]) < 1e-6
        assert abs((loss(x, gamma, beta + e) - loss(x, gamma, beta - e)) / (2 * h) - db[j]) < 1e-6
    z = np.linspace(-6, 6, 97)
    assert np.max(np.abs((O.gelu_from_erfc(z + h) - O.gelu_from_erfc(z - h)) / (2 * h) - O.gelu_slope(z))) < 1e-8
    assert np.max(np.abs(O.gelu_from_erfc(z) - O.gelu(z))) < 1e-14
