"""A transformer layer's normalisation and its 8-bit path, as measurable cases.

Six operators, each as one pass of a user's program over the k local tensors of its global tensors:

  layer_norm            y, mean and 1 / deviation of rows
  layer_norm_backward   gradients of the rows and, reduced over them, of gamma and beta
  quantize8             8-bit blocks of a tensor: e4m3 values, a power-of-two scale for each block of 128
                        (of 128 x 128 for weights), as stored or transposed
  gelu_save8            GeLU whose input is kept for the backward pass in 8-bit blocks
  gelu_save8_backward   gradient through GeLU from that 8-bit checkpoint
  matmul8               product of two 8-bit operands with a scale for each block

Where `own` is false run() is elementary torch in fp32, rounded once; where it is true it calls the library.
"""
import math

import numpy as np
import torch

own = False

F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
_DTYPE = {"f32": F32, "bf16": BF16}
BLOCK = 128
EPS = 1e-5


def listed():
    return [
        # a few sequences' next tokens through a small layer: the call is latency
        {"name": "norm_small", "op": "layer_norm", "rows": 64, "cols": 512, "dtype": "bf16", "shards": 2},
        # the activations of a training batch, split by rows over eight devices
        {"name": "norm_block", "op": "layer_norm", "rows": 8192, "cols": 4096, "dtype": "bf16", "shards": 8},
        # their gradient; the weights' gradients are wanted whole on every device (data parallelism)
        {"name": "norm_grad_block", "op": "layer_norm_backward", "rows": 8192, "cols": 4096, "dtype": "bf16", "shards": 8, "grads": "B"},
        # fp32 rows of odd length over three devices, the weights' gradients left as partial sums
        {"name": "norm_grad_ragged", "op": "layer_norm_backward", "rows": 1021, "cols": 1537, "dtype": "f32", "shards": 3, "grads": "P"},
        # activations on their way into an 8-bit product
        {"name": "quantize_tokens", "op": "quantize8", "rows": 8192, "cols": 4096, "dtype": "bf16", "shards": 8, "split": 0,
         "tiles": False, "transposed": False},
        # a layer's weight after its update, for the forward product: transposed, a scale a tile
        {"name": "quantize_weight", "op": "quantize8", "rows": 4096, "cols": 16384, "dtype": "bf16", "shards": 8, "split": 1,
         "tiles": True, "transposed": True},
        # the hidden layer of an MLP in training, its columns split over eight devices
        {"name": "gelu_save_block", "op": "gelu_save8", "rows": 8192, "cols": 16384, "dtype": "bf16", "shards": 8, "split": 1},
        # the same for a few rows
        {"name": "gelu_save_small", "op": "gelu_save8", "rows": 16, "cols": 16384, "dtype": "bf16", "shards": 8, "split": 1},
        # the way back through the hidden layer
        {"name": "gelu_grad_block", "op": "gelu_save8_backward", "rows": 8192, "cols": 16384, "dtype": "bf16", "shards": 8, "split": 1},
        # fp32 with rows of odd length
        {"name": "gelu_grad_ragged", "op": "gelu_save8_backward", "rows": 1021, "cols": 1537, "dtype": "f32", "shards": 3, "split": 0},
        # a few sequences that each add one token: the 8-bit weight is the traffic
        {"name": "product_decode", "op": "matmul8", "m": 16, "n": 16384, "k": 4096, "out": "bf16", "shards": 8, "sig": "columns"},
        # the same layer on a long prompt or a training batch
        {"name": "product_prefill", "op": "matmul8", "m": 8192, "n": 16384, "k": 4096, "out": "bf16", "shards": 8, "sig": "columns"},
    ]


def _log(rng, lo, hi, step=1):
    """A multiple of `step` between lo and hi, spread over the logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return int(min(hi, max(lo, round(v / step) * step)))


def draw(rng):
    op = rng.choice(["layer_norm", "layer_norm_backward", "quantize8", "gelu_save8", "gelu_save8_backward", "matmul8", "matmul8"])
    shards = rng.choice([1, 2, 3, 4, 8])
    if op == "matmul8":
        # widths of real layers are multiples of 16, which is what a row of 8-bit values needs to be read in whole vectors;
        # now and then one that is not
        step = rng.choice([64, 16, 16, 1])
        return {"op": op, "m": _log(rng, 1, 8192), "n": _log(rng, 128, 16384, step), "k": _log(rng, 128, 8192, step),
                "out": rng.choice(["bf16", "bf16", "f32"]), "shards": shards, "sig": rng.choice(["rows", "columns", "contraction"])}
    rows, cols = _log(rng, 1, 8192), _log(rng, 64, 16384)
    if rng.random() < 0.5:            # aligned rows, as most layers have them
        cols = max(64, cols // 64 * 64)
    c = {"op": op, "rows": rows, "cols": cols, "dtype": rng.choice(["f32", "bf16", "bf16"]), "shards": shards}
    if op == "layer_norm_backward":
        c["grads"] = rng.choice(["P", "B", "S0"])
    if op in ("quantize8", "gelu_save8", "gelu_save8_backward"):
        c["split"] = rng.choice([0, 1])
    if op == "quantize8":
        c["tiles"], c["transposed"] = rng.choice([(False, False), (False, True), (True, False), (True, True)])
    return c


# ------------------------------------------------------------------ layouts

def _parts(n, k):
    """(start, length) of the k pieces of a balanced split."""
    return [(r * (n // k) + min(r, n % k), n // k + (1 if r < n % k else 0)) for r in range(k)]


def _cut(t, axis, k):
    """Local tensors of t under a split along `axis`."""
    return [t.narrow(axis, s, n).contiguous() for s, n in _parts(t.shape[axis], k)]


def _blocks(n):
    return -(-n // BLOCK)


def _scales_like(values, tiles):
    """Room for the scales of local 8-bit tensors."""
    return [torch.empty(_blocks(v.shape[0]) if tiles else v.shape[0], _blocks(v.shape[1]), dtype=F32, device="cuda") for v in values]


# ------------------------------------------------------------------ 8-bit blocks, plain

def _power(e):
    """2^e for integers in [-126, 127], exactly."""
    return ((e + 127) << 23).view(F32)


def _exponents(amax):
    """The smallest e in [-126, ..] with amax <= 448 * 2^e; 0 for a block of zeros."""
    m, ex = torch.frexp(amax)
    e = torch.where(m <= 0.875, ex - 9, ex - 8).to(torch.int32).clamp(min=-126)
    return torch.where(amax > 0, e, torch.zeros_like(e))


def _spread(s, tiles, rows, cols):
    """One number per element from one per block."""
    s = s.repeat_interleave(BLOCK, 1)[:, :cols]
    return s.repeat_interleave(BLOCK, 0)[:rows] if tiles else s


def _quantize(x, tiles):
    """(e4m3 values, fp32 scales) of a matrix: blocks of 128 along its rows, or of 128 x 128."""
    x = x.float()
    rows, cols = x.shape
    mag = torch.where(torch.isfinite(x), x, torch.zeros_like(x)).abs()
    pad_r = _blocks(rows) * BLOCK - rows if tiles else 0
    mag = torch.nn.functional.pad(mag, (0, _blocks(cols) * BLOCK - cols, 0, pad_r))
    mag = mag.view(mag.shape[0], _blocks(cols), BLOCK).amax(2)
    if tiles:
        mag = mag.view(_blocks(rows), BLOCK, _blocks(cols)).amax(1)
    e = _exponents(mag)
    return (x * _spread(_power(-e), tiles, rows, cols)).to(E4M3), _power(e)


def _dequantize(values, scales, tiles):
    return values.float() * _spread(scales, tiles, *values.shape)


# ------------------------------------------------------------------ inputs

def _normal(g, shape, std, dtype):
    return (torch.randn(shape, dtype=F32, device="cuda", generator=g) * std).to(dtype)


def prepare(case, seed):
    """Inputs and room for the outputs; where the library is called, also its descriptors of them and its workspace, which a
    program sets up once for the buffers it keeps."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": case, **_PREPARE[case["op"]](case, g)}
    if own:
        s["t"] = _DESCRIBE[case["op"]](case, s)
    return s


def _activations(case, g):
    """Rows with offsets and spreads of their own, a few columns far larger than the rest."""
    rows, cols = case["rows"], case["cols"]
    x = _normal(g, (rows, cols), 1.0, F32)
    x *= torch.exp(0.5 * torch.randn(rows, 1, device="cuda", generator=g))
    x[:, :: max(1, cols // 7)] *= 8.0
    return x


def _prepare_layer_norm(case, g):
    dt, k, cols = _DTYPE[case["dtype"]], case["shards"], case["cols"]
    x = _cut((_activations(case, g) + 0.5 * torch.randn(case["rows"], 1, device="cuda", generator=g)).to(dt), 0, k)
    s = {"x": x, "gamma": 1.0 + _normal(g, (cols,), 0.2, F32), "beta": _normal(g, (cols,), 0.2, F32),
         "y": [torch.empty_like(t) for t in x],
         "mean": [torch.empty(t.shape[0], dtype=F32, device="cuda") for t in x]}
    s["rstd"] = [torch.empty_like(t) for t in s["mean"]]
    return s


def _prepare_layer_norm_backward(case, g):
    s = _prepare_layer_norm(case, g)
    dt, k, cols = _DTYPE[case["dtype"]], case["shards"], case["cols"]
    s["grad_y"] = _cut(_normal(g, (case["rows"], cols), 0.1, dt), 0, k)
    # what the forward pass left behind
    s["mean"] = [t.double().mean(1).float() for t in s["x"]]
    s["rstd"] = [(t.double().var(1, unbiased=False) + EPS).rsqrt().float() for t in s["x"]]
    s["grad_x"] = s.pop("y")
    size = {"P": [cols] * k, "B": [cols], "S0": [n for _, n in _parts(cols, k)]}[case["grads"]]
    s["grad_gamma"] = [torch.empty(n, dtype=F32, device="cuda") for n in size]
    s["grad_beta"] = [torch.empty(n, dtype=F32, device="cuda") for n in size]
    return s


def _prepare_quantize8(case, g):
    x = _cut(_activations(case, g).to(_DTYPE[case["dtype"]]), case["split"], case["shards"])
    values = [torch.empty(tuple(t.shape[::-1]) if case["transposed"] else tuple(t.shape), dtype=E4M3, device="cuda") for t in x]
    return {"x": x, "values": values, "scales": _scales_like(values, case["tiles"])}


def _prepare_gelu_save8(case, g):
    z = _cut(_activations(case, g).to(_DTYPE[case["dtype"]]), case["split"], case["shards"])
    values = [torch.empty(t.shape, dtype=E4M3, device="cuda") for t in z]
    return {"z": z, "y": [torch.empty_like(t) for t in z], "values": values, "scales": _scales_like(values, False)}


def _prepare_gelu_save8_backward(case, g):
    dt, k = _DTYPE[case["dtype"]], case["shards"]
    saved = [_quantize(t, False) for t in _cut(_activations(case, g).to(dt), case["split"], k)]
    grad_y = _cut(_normal(g, (case["rows"], case["cols"]), 0.1, dt), case["split"], k)
    return {"values": [v for v, _ in saved], "scales": [t for _, t in saved], "grad_y": grad_y,
            "grad_z": [torch.empty_like(t) for t in grad_y]}


# signature of x, of w (stored [n, k], as its transpose), of y; the axis that splits each, None for one copy
_SIGS = {"rows": (0, None, 0), "columns": (None, 0, 1), "contraction": (1, 1, None)}


def _local(t, axis, k):
    return [t] if axis is None else _cut(t, axis, k)


def _prepare_matmul8(case, g):
    m, n, kk, k = case["m"], case["n"], case["k"], case["shards"]
    ax, aw, ay = _SIGS[case["sig"]]
    x = _normal(g, (m, kk), 1.0, F32) * torch.exp(0.5 * torch.randn(m, 1, device="cuda", generator=g))
    x[:, :: max(1, kk // 7)] *= 8.0
    x = [_quantize(t, False) for t in _local(x, ax, k)]
    w = [_quantize(t, True) for t in _local(_normal(g, (n, kk), kk ** -0.5, F32), aw, k)]
    y = [torch.empty_like(t) for t in _local(torch.empty(m, n, dtype=_DTYPE[case["out"]], device="cuda"), ay, k)]
    return {"x": [v for v, _ in x], "x_scales": [t for _, t in x], "w": [v for v, _ in w], "w_scales": [t for _, t in w], "y": y}


_PREPARE = {"layer_norm": _prepare_layer_norm, "layer_norm_backward": _prepare_layer_norm_backward, "quantize8": _prepare_quantize8,
            "gelu_save8": _prepare_gelu_save8, "gelu_save8_backward": _prepare_gelu_save8_backward, "matmul8": _prepare_matmul8}


# ------------------------------------------------------------------ the library's descriptors

def _global(shape, axis, locals_, k):
    """The global tensor of the local tensors: split along `axis`; None: one buffer that is every replica; "P": partial sums."""
    import paper_2110_15032_b200 as sbp
    sig = sbp.B if axis is None else sbp.P_SUM if axis == "P" else sbp.S(axis)
    return sbp.SbpTensor(shape, locals_[0].dtype, sig, locals_ * k if axis is None else locals_)


def _joined(locals_, axis, k):
    """_global() of matrices or vectors whose global extent along `axis` is the sum of the local ones."""
    shape = list(locals_[0].shape)
    if axis is not None:
        shape[axis] = sum(t.shape[axis] for t in locals_)
    return _global(shape, axis, locals_, k)


def _describe_layer_norm(case, s):
    k = case["shards"]
    t = {n: _joined(s[n], 0, k) for n in ("x", "y", "mean", "rstd") if n in s}
    return {**t, "gamma": _joined([s["gamma"]], None, k), "beta": _joined([s["beta"]], None, k)}


def _describe_layer_norm_backward(case, s):
    import paper_2110_15032_b200 as sbp
    k, axis = case["shards"], {"P": "P", "B": None, "S0": 0}[case["grads"]]
    t = {**_describe_layer_norm(case, s), "grad_y": _joined(s["grad_y"], 0, k), "grad_x": _joined(s["grad_x"], 0, k)}
    for n in ("grad_gamma", "grad_beta"):
        t[n] = _global((case["cols"],), axis, s[n], k)
    t["ws"] = torch.empty(max(1, sbp.sbp_layer_norm_backward_workspace_bytes(t["x"])), dtype=torch.uint8, device="cuda")
    return t


def _describe_quantize8(case, s):
    axis = 1 - case["split"] if case["transposed"] else case["split"]
    return {"x": _joined(s["x"], case["split"], case["shards"]), "values": _joined(s["values"], axis, case["shards"]),
            "scales": _joined(s["scales"], axis, case["shards"])}


def _describe_gelu_save8(case, s):
    return {n: _joined(s[n], case["split"], case["shards"]) for n in ("z", "y", "values", "scales", "grad_y", "grad_z") if n in s}


def _describe_matmul8(case, s):
    ax, aw, ay = _SIGS[case["sig"]]
    return {n: _joined(s[n], a, case["shards"]) for n, a in (("x", ax), ("x_scales", ax), ("w", aw), ("w_scales", aw), ("y", ay))}


_DESCRIBE = {"layer_norm": _describe_layer_norm, "layer_norm_backward": _describe_layer_norm_backward, "quantize8": _describe_quantize8,
             "gelu_save8": _describe_gelu_save8, "gelu_save8_backward": _describe_gelu_save8, "matmul8": _describe_matmul8}


# ------------------------------------------------------------------ one pass

def run(state):
    return (_CALL if own else _PLAIN)[state["case"]["op"]](state["case"], state)


def _call_layer_norm(case, s):
    import paper_2110_15032_b200 as sbp
    t = s["t"]
    sbp.sbp_layer_norm(t["x"], t["gamma"], t["beta"], t["y"], t["mean"], t["rstd"], EPS)
    return s["y"] + s["mean"] + s["rstd"]


def _call_layer_norm_backward(case, s):
    import paper_2110_15032_b200 as sbp
    t = s["t"]
    sbp.sbp_layer_norm_backward(t["x"], t["gamma"], t["mean"], t["rstd"], t["grad_y"], t["grad_x"], t["grad_gamma"], t["grad_beta"], t["ws"])
    return s["grad_x"] + s["grad_gamma"] + s["grad_beta"]


def _call_quantize8(case, s):
    import paper_2110_15032_b200 as sbp
    t = s["t"]
    sbp.sbp_quantize8(t["x"], t["values"], t["scales"],
                      (sbp.SBP_QUANT_TILES if case["tiles"] else 0) | (sbp.SBP_TRANS_X if case["transposed"] else 0))
    return s["values"] + s["scales"]


def _call_gelu_save8(case, s):
    import paper_2110_15032_b200 as sbp
    t = s["t"]
    sbp.sbp_gelu_save8(t["z"], t["y"], t["values"], t["scales"])
    return s["y"] + s["values"] + s["scales"]


def _call_gelu_save8_backward(case, s):
    import paper_2110_15032_b200 as sbp
    t = s["t"]
    sbp.sbp_gelu_save8_backward(t["values"], t["scales"], t["grad_y"], t["grad_z"])
    return s["grad_z"]


def _call_matmul8(case, s):
    import paper_2110_15032_b200 as sbp
    t = s["t"]
    sbp.sbp_matmul8(t["x"], t["x_scales"], t["w"], t["w_scales"], t["y"])
    return s["y"]


_CALL = {"layer_norm": _call_layer_norm, "layer_norm_backward": _call_layer_norm_backward, "quantize8": _call_quantize8,
         "gelu_save8": _call_gelu_save8, "gelu_save8_backward": _call_gelu_save8_backward, "matmul8": _call_matmul8}


def _norm(x, gamma, beta):
    v = x.float()
    n = v.shape[1]
    mean = v.sum(1, keepdim=True) / n
    d = v - mean
    rstd = 1.0 / torch.sqrt((d * d).sum(1, keepdim=True) / n + EPS)
    return (d * rstd * gamma + beta).to(x.dtype), mean[:, 0], rstd[:, 0]


def _plain_layer_norm(case, s):
    out = [_norm(x, s["gamma"], s["beta"]) for x in s["x"]]
    return [o[0] for o in out] + [o[1] for o in out] + [o[2] for o in out]


def _norm_grad(x, mean, rstd, gamma, grad_y):
    rstd, dy, n = rstd[:, None], grad_y.float(), x.shape[1]
    h = (x.float() - mean[:, None]) * rstd
    a = dy * gamma
    dx = rstd * (a - a.sum(1, keepdim=True) / n - h * ((a * h).sum(1, keepdim=True) / n))
    return dx.to(x.dtype), (dy * h).sum(0), dy.sum(0)


def _shared(parts, grads, k):
    """Gradients of gamma or beta, one a device, as the case asks for them."""
    if grads == "P":
        return parts
    whole = torch.stack(parts).sum(0)
    return [whole] if grads == "B" else _cut(whole, 0, k)


def _plain_layer_norm_backward(case, s):
    out = [_norm_grad(x, m, r, s["gamma"], dy) for x, m, r, dy in zip(s["x"], s["mean"], s["rstd"], s["grad_y"])]
    k = case["shards"]
    return [o[0] for o in out] + _shared([o[1] for o in out], case["grads"], k) + _shared([o[2] for o in out], case["grads"], k)


def _plain_quantize8(case, s):
    out = [_quantize(x.t() if case["transposed"] else x, case["tiles"]) for x in s["x"]]
    return [v for v, _ in out] + [t for _, t in out]


def _gelu(z):
    v = z.float()
    return (0.5 * v * torch.special.erfc(v * -math.sqrt(0.5))).to(z.dtype)


def _plain_gelu_save8(case, s):
    out = [_quantize(z, False) for z in s["z"]]
    return [_gelu(z) for z in s["z"]] + [v for v, _ in out] + [t for _, t in out]


def _gelu_grad(values, scales, grad_y):
    z = _dequantize(values, scales, False)
    slope = 0.5 * torch.special.erfc(z * -math.sqrt(0.5)) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    return (grad_y.float() * slope).to(grad_y.dtype)


def _plain_gelu_save8_backward(case, s):
    return [_gelu_grad(v, t, dy) for v, t, dy in zip(s["values"], s["scales"], s["grad_y"])]


def _plain_matmul8(case, s):
    _, aw, ay = _SIGS[case["sig"]]
    dt, k = _DTYPE[case["out"]], case["shards"]
    x = [_dequantize(v, t, False) for v, t in zip(s["x"], s["x_scales"])]
    w = [_dequantize(v, t, True) for v, t in zip(s["w"], s["w_scales"])]
    if ay is None:                     # partial products, summed
        return [torch.stack([torch.matmul(a, b.t()) for a, b in zip(x, w)]).sum(0).to(dt)]
    x, w = x * (k // len(x)), w * (k // len(w))
    return [torch.matmul(a, b.t()).to(dt) for a, b in zip(x, w)]


_PLAIN = {"layer_norm": _plain_layer_norm, "layer_norm_backward": _plain_layer_norm_backward, "quantize8": _plain_quantize8,
          "gelu_save8": _plain_gelu_save8, "gelu_save8_backward": _plain_gelu_save8_backward, "matmul8": _plain_matmul8}


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    op = case["op"]
    if op == "matmul8":
        m, n, kk, k = case["m"], case["n"], case["k"], case["shards"]
        out = 2 if case["out"] == "bf16" else 4
        scales = m * _blocks(kk) + _blocks(n) * _blocks(kk)
        return {"bytes": m * kk + n * kk + 4 * scales + out * m * n, "flops": 2 * m * n * kk}
    rows, cols, e = case["rows"], case["cols"], 2 if case["dtype"] == "bf16" else 4
    n = rows * cols
    if op == "layer_norm":
        return {"bytes": 2 * n * e + 8 * cols + 8 * rows, "flops": 8 * n}
    if op == "layer_norm_backward":
        copies = case["shards"] if case["grads"] == "P" else 1
        return {"bytes": 3 * n * e + 4 * cols + 8 * rows + 8 * cols * copies, "flops": 14 * n}
    scales = 4 * n // BLOCK
    if op == "quantize8":
        return {"bytes": n * (e + 1) + (scales // BLOCK if case["tiles"] else scales), "flops": 3 * n}
    return {"bytes": n * (2 * e + 1) + scales, "flops": 25 * n}


# ------------------------------------------------------------------ the definitions in 64 bits

def exact(case, seed):
    if case["op"] == "matmul8" and 2.0 * case["m"] * case["n"] * case["k"] > 1e14:
        return None
    g = torch.Generator(device="cuda").manual_seed(seed)
    return _EXACT[case["op"]](case, _PREPARE[case["op"]](case, g))


def _exact_layer_norm(case, s):
    gamma, beta = s["gamma"].double(), s["beta"].double()
    x = [t.double() for t in s["x"]]
    mean = [t.mean(1) for t in x]
    rstd = [((t - m[:, None]).pow(2).mean(1) + EPS).pow(-0.5) for t, m in zip(x, mean)]
    return [(t - m[:, None]) * r[:, None] * gamma + beta for t, m, r in zip(x, mean, rstd)] + mean + rstd


def _exact_layer_norm_backward(case, s):
    gamma, k = s["gamma"].double(), case["shards"]
    dx, dg, db = [], [], []
    for x, mean, rstd, dy in zip(s["x"], s["mean"], s["rstd"], s["grad_y"]):
        xhat = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
        dy = dy.double()
        weighted = dy * gamma
        dx.append(rstd.double()[:, None] * (weighted - weighted.mean(1, keepdim=True) - xhat * (weighted * xhat).mean(1, keepdim=True)))
        dg.append((dy * xhat).sum(0))
        db.append(dy.sum(0))
    if case["grads"] != "P":
        dg, db = [sum(dg)], [sum(db)]
        if case["grads"] == "S0":
            dg, db = _cut(dg[0], 0, k), _cut(db[0], 0, k)
    return dx + dg + db


def _exact_blocks(x, tiles):
    """Values and scales of a host matrix in float64: block maxima by numpy, steps of e4m3 from the exponent of each number."""
    rows, cols = x.shape
    height = BLOCK if tiles else 1
    big = np.maximum.reduceat(np.abs(x), np.arange(0, cols, BLOCK), axis=1)
    big = np.maximum.reduceat(big, np.arange(0, rows, height), axis=0)
    safe = np.where(big > 0, big, 448.0)
    e = np.floor(np.log2(safe)) - 9.0                       # below the answer by one or two
    for _ in range(3):
        e = np.where(safe > 448.0 * np.exp2(e), e + 1.0, e)
    e = np.maximum(e, -126.0)
    scales = np.exp2(e)
    per = np.repeat(np.repeat(scales, BLOCK, 1)[:, :cols], height, 0)[:rows]
    v = x / per
    step = np.exp2(np.maximum(np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -200))), -6.0) - 3.0)
    return torch.from_numpy(np.rint(v / step) * step), torch.from_numpy(scales)


def _exact_quantize8(case, s):
    if case["rows"] * case["cols"] > 1 << 24:               # minutes of numpy: the answer has no rounding of its own to judge
        return None
    out = [_exact_blocks((x.t() if case["transposed"] else x).double().cpu().numpy(), case["tiles"]) for x in s["x"]]
    return [v for v, _ in out] + [t for _, t in out]


def _exact_gelu_save8(case, s):
    y = [z.double() * torch.special.ndtr(z.double()) for z in s["z"]]
    if case["rows"] * case["cols"] > 1 << 24:
        return y + [None] * (2 * case["shards"])
    out = [_exact_blocks(z.double().cpu().numpy(), False) for z in s["z"]]
    return y + [v for v, _ in out] + [t for _, t in out]


def _exact_gelu_save8_backward(case, s):
    out = []
    for v, t, dy in zip(s["values"], s["scales"], s["grad_y"]):
        column = torch.arange(v.shape[1], device="cuda") // BLOCK
        z = v.float().double() * t.double()[:, column]
        out.append(dy.double() * (torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)))
    return out


def _exact_matmul8(case, s):
    def whole(values, scales, axis, tiles):
        parts = []
        for v, t in zip(values, scales):
            column, row = torch.arange(v.shape[1], device="cuda") // BLOCK, torch.arange(v.shape[0], device="cuda")
            parts.append(v.float().double() * t.double()[row // BLOCK if tiles else row][:, column])
        return torch.cat(parts, axis or 0)

    ax, aw, ay = _SIGS[case["sig"]]
    y = whole(s["x"], s["x_scales"], ax, False) @ whole(s["w"], s["w_scales"], aw, True).t()
    return _local(y, ay, case["shards"])


_EXACT = {"layer_norm": _exact_layer_norm, "layer_norm_backward": _exact_layer_norm_backward, "quantize8": _exact_quantize8,
          "gelu_save8": _exact_gelu_save8, "gelu_save8_backward": _exact_gelu_save8_backward, "matmul8": _exact_matmul8}
