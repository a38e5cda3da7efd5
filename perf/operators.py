"""The work of the microscaled number formats, as cases that can be timed and compared.

A case is a dict of plain values; ``prepare`` makes what a user's program holds before the call, ``run`` makes one
pass, ``work`` says what that pass cannot do without, ``exact`` gives the pass's results in 64 bits.  With ``own`` the
pass goes through this library's entry points, without it the operators are written out in elementary tensor
operations in 32 bits, rounded once at the end.

Formats (a block is a run of consecutive elements of a row, the last one filled up with zeros):

``mxfp4``    32 elements of 4 bits (sign, 2 exponent bits, 1 fraction bit: 0 .5 1 1.5 2 3 4 6) and a power of two,
             2^(floor(log2 max|x|) - 2); elements rounded to nearest even, saturating at 6
``nvfp4``    16 such elements, a scale with 4 exponent and 3 fraction bits, and one fp32 scale per tensor that comes
             from the tensor's largest magnitude m: enc = 2688 / m, s = e4m3(max|x| * (448 / m)),
             q = e2m1(x * (enc / s)), value = q * s * (m / 2688)
``mxint8``   32 elements of 8 bits, q in -127..127 in units of 2^-6, and the power of two 2^floor(log2 max|x|)

Two 4-bit elements share a byte, the even one in its low half.  A row of codes takes its length rounded up to whole
blocks of 32.  The scales of the 4-bit formats lie in tiles of 128 rows x 4 scales: byte (r % 32) * 16 + (r % 128) /
32 * 4 + c % 4 of tile (r / 128, c / 4), tiles of a row block back to back.  Those of mxint8 lie row by row, each row
filled up to a multiple of 16.

Kinds: ``codec`` (a tensor to codes and back), ``linear`` (a layer's activations to 4 bits, times weights that are
already in 4 bits), ``product`` (both operands in 4 bits), ``act`` (an activation function whose input is kept in 8
bits), ``act_grad`` (its backward pass from the 8 bits), ``wgrad`` (a weight's gradient from an input kept in 8 bits).
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = {"mxfp4": 32, "nvfp4": 16, "mxint8": 32}
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # The activations of a few tokens, quantized and looked at again: latency of two launches.
        {"name": "codec-nvfp4-64x1024", "kind": "codec", "format": "nvfp4", "rows": 64, "cols": 1024, "dtype": "bf16"},
        # The activations of a large batch through 4 bits (quantization-aware training, error measurement).
        {"name": "codec-mxfp4-16384x4096", "kind": "codec", "format": "mxfp4", "rows": 16384, "cols": 4096,
         "dtype": "bf16"},
        # One token through a layer: the weights are read once.
        {"name": "linear-nvfp4-1x4096x4096", "kind": "linear", "format": "nvfp4", "m": 1, "n": 4096, "k": 4096,
         "dtype": "bf16", "relu": False},
        # A ragged batch and a layer whose sizes are no multiple of anything, with bias, ReLU and fp32 out.
        {"name": "linear-mxfp4-250x1001x1000", "kind": "linear", "format": "mxfp4", "m": 250, "n": 1001, "k": 1000,
         "dtype": "f32", "relu": True},
        # The repository's large fully connected layer, both operands at hand in 4 bits.
        {"name": "product-nvfp4-16384x4096x4096", "kind": "product", "format": "nvfp4", "m": 16384, "n": 4096,
         "k": 4096, "dtype": "bf16", "relu": False},
        # The feed-forward block's gate and up projections, side by side in one matrix, and its product.
        {"name": "act-silu-gated-8192x8192", "kind": "act", "act": "silu", "gated": True, "rows": 8192, "cols": 8192,
         "dtype": "bf16"},
        # A small fp32 tensor with rows of odd length.
        {"name": "act-gelu-333x1001", "kind": "act", "act": "gelu", "gated": False, "rows": 333, "cols": 1001,
         "dtype": "f32"},
        # The backward passes of the same.
        {"name": "act_grad-silu-gated-8192x8192", "kind": "act_grad", "act": "silu", "gated": True, "rows": 8192,
         "cols": 8192, "dtype": "bf16"},
        {"name": "act_grad-relu-77x2500", "kind": "act_grad", "act": "relu", "gated": False, "rows": 77,
         "cols": 2500, "dtype": "bf16"},
        # Weight gradient of the large fully connected layer.
        {"name": "wgrad-16384x4096x4096", "kind": "wgrad", "m": 16384, "n": 4096, "k": 4096},
        # Of a convolution layer as a product (the 28x28x128 maps of 128 images, 3x3): few outputs, a long sum.
        {"name": "wgrad-100352x128x1152", "kind": "wgrad", "m": 100352, "n": 128, "k": 1152},
        # A short last batch.
        {"name": "wgrad-333x200x1000", "kind": "wgrad", "m": 333, "n": 200, "k": 1000},
    ]


def _log(rng, lo, hi):
    """An integer of [lo, hi], spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["codec", "linear", "product", "act", "act_grad", "wgrad"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "codec":
        cols = _log(rng, 16, 8192)
        return {"kind": kind, "format": rng.choice(["mxfp4", "nvfp4", "mxint8"]), "rows": max(1, _log(rng, 1 << 14, 1 << 25) // cols),
                "cols": cols, "dtype": dtype}
    if kind in ("linear", "product"):
        lo, hi = (1, 2048) if kind == "linear" else (64, 16384)
        while True:
            c = {"kind": kind, "format": rng.choice(["mxfp4", "nvfp4"]), "m": _log(rng, lo, hi), "n": _log(rng, 64, 8192),
                 "k": _log(rng, 64, 8192), "dtype": dtype, "relu": rng.random() < 0.3}
            if c["m"] * c["n"] * c["k"] <= 1 << 37:
                return c
    if kind in ("act", "act_grad"):
        cols = _log(rng, 16, 8192)
        return {"kind": kind, "act": rng.choice(["silu", "gelu", "relu"]), "gated": rng.random() < 0.5,
                "rows": max(1, _log(rng, 1 << 14, 1 << 25) // cols), "cols": cols, "dtype": dtype}
    while True:
        c = {"kind": kind, "m": _log(rng, 16, 131072), "n": _log(rng, 8, 512) * 8, "k": _log(rng, 64, 4096)}
        if c["m"] * c["n"] * c["k"] <= 1 << 37:
            return c


# ---- the formats, in 32 bits --------------------------------------------------------------------

def _up(a, b):
    return -(-a // b) * b


def _pow2(e):
    """2.0 ** e for whole numbers e in -127..127, in fp32: the bits of its exponent, or of the one subnormal."""
    return torch.where(e > -127, (e.int() + 127) << 23, 1 << 22).view(torch.float32)


def _e2m1(v):
    """fp32 to the nearest of 0 .5 1 1.5 2 3 4 6, ties to the even code."""
    a = v.abs().clamp(max=6.0)
    step = torch.where(a < 2.0, 0.5, torch.where(a < 4.0, 1.0, 2.0))
    return torch.copysign(torch.round(a / step) * step, v)


def _floor_log2(a):
    return torch.where(a > 0, torch.frexp(a)[1] - 1, -200)


def _largest(m):
    """The tensor's largest magnitude as nvfp4 takes it."""
    return torch.where(m < 2.0 ** -100, torch.full_like(m, 2.0 ** -100), m)


def _quantize(x, fmt, m):
    """x (rows, cols) -> (elements (rows, blocks, block) as fp32 values, scale codes (rows, blocks) as uint8, scale
    values in fp32 without the tensor's own)."""
    rows, cols = x.shape
    b = BLOCK[fmt]
    x = torch.nn.functional.pad(x.float(), (0, _up(cols, 32) - cols)).view(rows, -1, b)
    a = x.abs().amax(-1)
    if fmt == "nvfp4":
        m = _largest(m)
        # a number over a tensor is its reciprocal times the number, which rounds twice
        s = (a * (torch.full_like(m, 448.0) / m)).clamp(max=448.0).to(torch.float8_e4m3fn)
        r = torch.where(s.float() > 0, (torch.full_like(m, 2688.0) / m) / s.float(), 0.0)
        return _e2m1(x * r[..., None]), s.view(torch.uint8), s.float()
    e = (_floor_log2(a) - (2 if fmt == "mxfp4" else 0)).clamp(min=-127)
    v = x * _pow2(-e)[..., None]
    q = _e2m1(v) if fmt == "mxfp4" else torch.round(v * 64.0).clamp(-127.0, 127.0)
    return q, (e + 127).to(torch.uint8), _pow2(e)


def _pack4(q):
    """Elements as values -> two codes a byte."""
    a = q.abs()
    code = (2.0 * a).where(a < 2.0, (a + 2.0).where(a < 4.0, a * 0.5 + 4.0)).to(torch.uint8)
    code = (code | (torch.signbit(q).to(torch.uint8) << 3)).flatten(1)
    return code[:, 0::2] | (code[:, 1::2] << 4)


def _tile_scales(s):
    """Scale codes (rows, blocks) -> tiles of 128 rows x 4."""
    r, c = s.shape
    s = torch.nn.functional.pad(s, (0, _up(c, 4) - c, 0, _up(r, 128) - r))
    return s.view(-1, 4, 32, _up(c, 4) // 4, 4).permute(0, 3, 2, 1, 4).contiguous().view(-1)


def _untile_scales(t, r, c):
    c4 = _up(c, 4) // 4
    return t.view(-1, c4, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(-1, c4 * 4)[:r, :c]


def _decode4(codes, scales, fmt):
    """Codes and tiled scales -> values in fp32 without the tensor's own scale."""
    table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
    b, rows = BLOCK[fmt], codes.shape[0]
    q = table[torch.stack([codes & 15, codes >> 4], -1).int()].view(rows, -1, b)
    s = _untile_scales(scales, rows, q.shape[1])
    s = s.contiguous().view(torch.float8_e4m3fn).float() if fmt == "nvfp4" else _pow2(s.int() - 127)
    return (q * s[..., None]).flatten(1)


def _decode8(codes, scales, cols):
    """mxint8 codes (rows, length) and scales (rows, length) -> fp32 (rows, cols)."""
    rows = codes.shape[0]
    q = codes.float().view(rows, -1, 32) * 2.0 ** -6
    return (q * _pow2(scales[:, :q.shape[1]].int() - 127)[..., None]).flatten(1)[:, :cols]


def _rows16(s):
    return torch.nn.functional.pad(s, (0, _up(s.shape[1], 16) - s.shape[1]))


# ---- inputs --------------------------------------------------------------------------------------

def _activations(g, rows, cols, dtype):
    """A layer's inputs: normal, channels of different size, a few of them large."""
    channel = torch.exp(0.5 * torch.randn(cols, generator=g, device="cuda"))
    channel = torch.where(torch.rand(cols, generator=g, device="cuda") < 0.01, channel * 12.0, channel)
    return (torch.randn((rows, cols), generator=g, device="cuda") * channel).to(dtype)


def _operand(x, fmt):
    """A matrix in 4 bits, as quantization leaves it."""
    m = x.float().abs().amax().view(1)
    q, s, _ = _quantize(x, fmt, m)
    return {"codes": _pack4(q), "scales": _tile_scales(s), "max": m}


def _kept(x):
    """A tensor in 8 bits, as an earlier forward pass leaves it."""
    q, s, _ = _quantize(x, "mxint8", None)
    return {"codes": q.flatten(1).to(torch.int8), "scales": _rows16(s)}


def _empty(fmt, rows, cols):
    """Room for the codes and scales of a tensor."""
    n, new = _up(cols, 32), lambda *s, dt=torch.uint8: torch.empty(s, dtype=dt, device="cuda")
    if fmt == "mxint8":
        return {"codes": new(rows, n, dt=torch.int8), "scales": new(rows, _up(n // 32, 16))}
    return {"codes": new(rows, n // 2), "scales": new(_up(rows, 128) * _up(n // BLOCK[fmt], 4))}


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    kind, s = case["kind"], dict(case)
    if kind == "codec":
        x = _activations(g, case["rows"], case["cols"], DTYPES[case["dtype"]])
        s.update(x=x, max=x.float().abs().amax().view(1), kept=_empty(case["format"], *x.shape), out=torch.empty_like(x))
    elif kind in ("linear", "product"):
        m, n, k = case["m"], case["n"], case["k"]
        x = _activations(g, m, k, torch.bfloat16)
        w = torch.randn((n, k), generator=g, device="cuda") * k ** -0.5
        s.update(w=_operand(w, case["format"]), bias=torch.randn(n, generator=g, device="cuda") if kind == "linear" else None,
                 out=torch.empty((m, n), dtype=DTYPES[case["dtype"]], device="cuda"))
        if kind == "linear":    # the largest magnitude comes from an earlier calibration
            s.update(x=x, max=x.float().abs().amax().view(1), a=_empty(case["format"], m, k))
        else:
            s["a"] = _operand(x, case["format"])
    elif kind in ("act", "act_grad"):
        rows, cols, dt = case["rows"], case["cols"], DTYPES[case["dtype"]]
        wide = torch.randn((rows, cols * (2 if case["gated"] else 1)), generator=g, device="cuda").mul_(2.0).to(dt)
        x, up = wide[:, :cols], wide[:, cols:] if case["gated"] else None
        if kind == "act":
            s.update(x=x, up=up, y=torch.empty((rows, cols), dtype=dt, device="cuda"), kept=_empty("mxint8", rows, cols),
                     up_kept=_empty("mxint8", rows, cols) if case["gated"] else None)
        else:
            dy = torch.randn((rows, cols), generator=g, device="cuda").mul_(1e-3).to(dt)
            d = torch.empty_like(wide)
            s.update(kept=_kept(x), up_kept=_kept(up) if case["gated"] else None, dy=dy, dx=d[:, :cols],
                     dup=d[:, cols:] if case["gated"] else None)
    else:
        m, n, k = case["m"], case["n"], case["k"]
        dy = torch.randn((m, n), generator=g, device="cuda").mul_(1e-3).to(torch.bfloat16)
        s.update(kept=_kept(_activations(g, m, k, torch.bfloat16)), dy=dy, dw=torch.empty((n, k), device="cuda"))
    return s


# ---- one pass ------------------------------------------------------------------------------------

def _sigmoid(x):
    return 1.0 / (1.0 + torch.exp(-x))


def _act(x, act):
    """The function and its derivative, in 32 bits."""
    if act == "relu":
        return torch.where(x > 0, x, 0.0), torch.where(x > 0, 1.0, 0.0)
    if act == "silu":
        s = _sigmoid(x)
        return x * s, s + x * s * (1.0 - s)
    c, a = 2.0 * math.sqrt(2.0 / math.pi), 0.044715      # gelu with tanh: x * sigmoid(2 sqrt(2 / pi) (x + a x^3))
    s = _sigmoid(c * (x + a * x * x * x))
    return x * s, s + x * s * (1.0 - s) * (c + 3.0 * a * c * x * x)


def _plain(s):
    kind = s["kind"]
    if kind == "codec":
        x, fmt = s["x"], s["format"]
        q, _, scale = _quantize(x, fmt, s["max"])
        v = (q * (2.0 ** -6 if fmt == "mxint8" else 1.0) * scale[..., None]).flatten(1)[:, :x.shape[1]]
        v = v * (_largest(s["max"]) / 2688.0) if fmt == "nvfp4" else v
        return {"values": v.to(x.dtype)}
    if kind in ("linear", "product"):
        fmt, w = s["format"], s["w"]
        if kind == "linear":
            q, _, scale = _quantize(s["x"], fmt, s["max"])
            a, am = (q * scale[..., None]).flatten(1), s["max"]
        else:
            a, am = _decode4(s["a"]["codes"], s["a"]["scales"], fmt), s["a"]["max"]
        y = a @ _decode4(w["codes"], w["scales"], fmt).T
        y = y * ((_largest(am) / 2688.0) * (_largest(w["max"]) / 2688.0)) if fmt == "nvfp4" else y
        y = y + s["bias"] if s["bias"] is not None else y
        return {"out": (torch.where(y > 0, y, 0.0) if s["relu"] else y).to(s["out"].dtype)}
    if kind == "act":
        y = _act(s["x"].float(), s["act"])[0]
        got = {"y": (y * s["up"].float() if s["gated"] else y).to(s["x"].dtype)}
        q, scale, _ = _quantize(s["x"], "mxint8", None)
        got.update(codes=q.flatten(1).to(torch.int8), scales=_rows16(scale))
        if s["gated"]:
            q, scale, _ = _quantize(s["up"], "mxint8", None)
            got.update(up_codes=q.flatten(1).to(torch.int8), up_scales=_rows16(scale))
        return got
    if kind == "act_grad":
        dy, cols = s["dy"].float(), s["dy"].shape[1]
        y, d = _act(_decode8(s["kept"]["codes"], s["kept"]["scales"], cols), s["act"])
        if not s["gated"]:
            return {"dx": (dy * d).to(s["dy"].dtype)}
        up = _decode8(s["up_kept"]["codes"], s["up_kept"]["scales"], cols)
        return {"dx": (dy * up * d).to(s["dy"].dtype), "dup": (dy * y).to(s["dy"].dtype)}
    return {"dw": s["dy"].float().T @ _decode8(s["kept"]["codes"], s["kept"]["scales"], s["dw"].shape[1])}


def run(s):
    if not own:
        return _plain(s)
    import paper_2105_11010_b200 as sparq
    kind = s["kind"]
    fmt = {"mxfp4": sparq.FORMAT_MXFP4, "nvfp4": sparq.FORMAT_NVFP4, "mxint8": sparq.FORMAT_MXINT8}[s.get("format", "mxint8")]
    if kind == "codec":
        k, m = s["kept"], s["max"] if s["format"] == "nvfp4" else None
        sparq.sparq_quantize_mx(s["x"], fmt, k["codes"], k["scales"], max_dev=m)
        sparq.sparq_dequantize_mx(k["codes"], k["scales"], fmt, s["out"], max_dev=m)
        return {"values": s["out"]}
    if kind in ("linear", "product"):
        a, w = s["a"], s["w"]
        am, wm = (s["max"] if kind == "linear" else a["max"], w["max"]) if s["format"] == "nvfp4" else (None, None)
        if kind == "linear":
            sparq.sparq_quantize_mx(s["x"], fmt, a["codes"], a["scales"], max_dev=am)
        out = {"bf16_out" if s["dtype"] == "bf16" else "f32_out": s["out"]}
        sparq.sparq_gemm_mxf4(a["codes"], a["scales"], w["codes"], w["scales"], fmt, a_max=am, b_max=wm, bias=s["bias"], relu=s["relu"], **out)
        return {"out": s["out"]}
    act = {"relu": sparq.ACT_RELU, "silu": sparq.ACT_SILU, "gelu": sparq.ACT_GELU}.get(s.get("act"))
    if kind == "act":
        k, u = s["kept"], s["up_kept"] or {}
        sparq.sparq_act_forward_mx8(s["x"], act, s["y"], k["codes"], k["scales"], up=s["up"], up_codes=u.get("codes"), up_scales=u.get("scales"))
        return {"y": s["y"], **k, **{"up_" + n: t for n, t in u.items()}}
    if kind == "act_grad":
        k, u = s["kept"], s["up_kept"] or {}
        sparq.sparq_act_backward_mx8(s["dy"], k["codes"], k["scales"], act, s["dx"], up_codes=u.get("codes"), up_scales=u.get("scales"), dup=s["dup"])
        return {"dx": s["dx"], "dup": s["dup"]} if s["gated"] else {"dx": s["dx"]}
    sparq.sparq_wgrad_mx8(s["dy"], s["kept"]["codes"], s["kept"]["scales"], s["dw"])
    return {"dw": s["dw"]}


# ---- what a pass cannot do without -----------------------------------------------------------------

def work(case):
    kind = case["kind"]
    width = 2 if case.get("dtype", "bf16") == "bf16" else 4
    if kind == "codec":     # values in and out; codes and scales out and in
        n = _up(case["cols"], 32)
        code = n + n // 32 if case["format"] == "mxint8" else n // 2 + n // BLOCK[case["format"]]
        return {"bytes": 2 * case["rows"] * (case["cols"] * width + code), "flops": 0}
    if kind in ("linear", "product"):
        m, n, k = case["m"], case["n"], case["k"]
        row = _up(k, 32) // 2 + _up(k, 32) // BLOCK[case["format"]]
        rest = m * n * width + (4 * n if kind == "linear" else 0)
        return {"bytes": (m + n) * row + rest + (2 * m * k + m * row if kind == "linear" else 0), "flops": 2.0 * m * n * k}
    if kind in ("act", "act_grad"):
        n, tensors = _up(case["cols"], 32), 2 if case["gated"] else 1
        plain, coded = case["rows"] * case["cols"] * width, case["rows"] * (n + n // 32)
        return {"bytes": (tensors + 1) * plain + tensors * coded, "flops": 0}
    m, n, k = case["m"], case["n"], case["k"]
    return {"bytes": 2 * m * n + m * (_up(k, 32) + _up(k, 32) // 32) + 4 * n * k, "flops": 2.0 * m * n * k}


# ---- in 64 bits, from the definitions --------------------------------------------------------------

GRID4 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
# Halfway points of GRID4, and whether a value on one goes up: to the code whose last bit is 0.
HALF4 = ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False))


def _x_nearest4(v):
    index = torch.zeros(v.shape, dtype=torch.long, device=v.device)
    for border, up in HALF4:
        index += (v.abs() >= border) if up else (v.abs() > border)
    return torch.tensor(GRID4, dtype=torch.float64, device=v.device)[index] * torch.where(v < 0, -1.0, 1.0)


def _x_binade(v):
    """The power of two at or below a positive 64-bit value, by its exponent bits (a logarithm may miss by one)."""
    return ((v.contiguous().view(torch.int64) >> 52) << 52).view(torch.float64)


def _x_f32(v):
    """A 64-bit result rounded to 32 where the format says so."""
    return v.to(torch.float32).to(torch.float64)


def _x_through(x, fmt, largest=None):
    """What a tensor's codes stand for, in 64 bits."""
    cols, b = x.shape[1], BLOCK[fmt]
    x = torch.cat([x.double(), x.new_zeros((x.shape[0], -x.shape[1] % b), dtype=torch.float64)], 1).unflatten(1, (-1, b))
    top = x.abs().max(-1, keepdim=True)[0]
    if fmt == "nvfp4":
        largest = largest.double().clamp(min=2.0 ** -100)
        s = _x_f32(top * _x_f32(448.0 / largest)).clamp(max=448.0)
        # e4m3: 4 significant bits down to 2^-6, steps of 2^-9 below
        step = _x_binade(s.clamp(min=2.0 ** -6)) / 8.0
        s = torch.round(s / step) * step
        r = torch.where(s > 0, _x_f32(_x_f32(2688.0 / largest) / s.clamp(min=2.0 ** -9)), 0.0)
        return (_x_nearest4(_x_f32(x * r)) * s * (largest / 2688.0)).flatten(1)[:, :cols]
    scale = (_x_binade(top) / (4.0 if fmt == "mxfp4" else 1.0)).clamp(min=2.0 ** -127)
    v = x / scale
    q = _x_nearest4(v) if fmt == "mxfp4" else torch.round(v * 64.0).clamp(-127.0, 127.0) / 64.0
    return (q * scale).flatten(1)[:, :cols]


def _x_read4(t, fmt, k):
    """What codes in memory stand for."""
    rows, b = t["codes"].shape[0], BLOCK[fmt]
    nibble = torch.stack([t["codes"] % 16, t["codes"] // 16], -1).flatten(1).long()
    v = torch.tensor(GRID4, dtype=torch.float64, device=nibble.device)[nibble % 8] * torch.where(nibble >= 8, -1.0, 1.0)
    r = torch.arange(rows, device=v.device)[:, None]
    c = torch.arange(v.shape[1] // b, device=v.device)[None, :]
    tiles = -(-(v.shape[1] // b) // 4)
    at = t["scales"][(r // 128 * tiles + c // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + c % 4].double()
    if fmt == "nvfp4":
        e, f = torch.floor(at / 8.0), at % 8
        s = torch.where(e == 0, f * 2.0 ** -9, (1.0 + f / 8.0) * torch.exp2(e - 7.0)) * (t["max"].double().clamp(min=2.0 ** -100) / 2688.0)
    else:
        s = torch.exp2(at - 127.0)
    return (v * s.repeat_interleave(b, 1))[:, :k]


def _x_read8(t, cols):
    s = torch.exp2(t["scales"].double() - 127.0 - 6.0)[:, :t["codes"].shape[1] // 32].repeat_interleave(32, 1)
    return (t["codes"].double() * s)[:, :cols]


def _x_act(x, act):
    if act == "relu":
        return x.clamp(min=0.0), (x > 0).double()
    z = x if act == "silu" else math.sqrt(8.0 / math.pi) * (x + 0.044715 * x ** 3)
    dz = 1.0 if act == "silu" else math.sqrt(8.0 / math.pi) * (1.0 + 3.0 * 0.044715 * x ** 2)
    p, n = torch.sigmoid(z), torch.sigmoid(-z)
    return x * p, p + x * p * n * dz


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "codec":
        return {"values": _x_through(s["x"], case["format"], s["max"])}
    if kind in ("linear", "product"):
        k, fmt = case["k"], case["format"]
        a = _x_through(s["x"], fmt, s["max"]) if kind == "linear" else _x_read4(s["a"], fmt, k)
        y = a @ _x_read4(s["w"], fmt, k).T
        y = y + s["bias"].double() if s["bias"] is not None else y
        return {"out": y.clamp(min=0.0) if case["relu"] else y}
    if kind == "act":       # the codes are whole numbers
        y = _x_act(s["x"].double(), case["act"])[0]
        return {"y": y * s["up"].double() if case["gated"] else y}
    if kind == "act_grad":
        dy = s["dy"].double()
        y, d = _x_act(_x_read8(s["kept"], case["cols"]), case["act"])
        if not case["gated"]:
            return {"dx": dy * d}
        return {"dx": dy * _x_read8(s["up_kept"], case["cols"]) * d, "dup": dy * y}
    return {"dw": s["dy"].double().T @ _x_read8(s["kept"], case["k"])}
