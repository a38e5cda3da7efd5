"""The elementwise microscaled kernels beyond one pass of their grid (19.4 million elements on 148 SMs), and in place on rows that are
no multiple of a vector: bit for bit what smaller calls, calls out of place and plain tensor operations give."""
import pytest
import torch

import mx_reference as ref
import paper_2105_11010_b200 as sparq

pytestmark = pytest.mark.gpu

FORMATS = [ref.MXFP4, ref.NVFP4, ref.MXINT8]
LARGE = [(3000, 8192), (5003, 4101), (600001, 37), (20000, 1000), (160001, 128)]          # aligned, odd, short, of 16 bytes, one run of scales
STEP = 1024                                                                                  # rows of a small call: whole blocks of scales


def tensor(seed, rows, cols, dtype, pitch=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((rows, pitch or cols), generator=g, device="cuda") * torch.exp(torch.randn((rows, 1), generator=g, device="cuda"))
    return x.to(dtype)[:, :cols]


def buffers(fmt, rows, cols):
    n = ref.up(cols, 32)
    codes = torch.full((rows, n if fmt == ref.MXINT8 else n // 2), 85, dtype=torch.int8 if fmt == ref.MXINT8 else torch.uint8, device="cuda")
    return codes, torch.full((sparq.sparq_mx_scale_bytes(fmt, rows, cols),), 85, dtype=torch.uint8, device="cuda")


def pieces(rows, cols):
    """Row ranges of a few small calls: the first, ones behind each pass of the grid, the last."""
    per_pass = 148 * 32 * 256 * 16 // ref.up(cols, 32)
    for first in sorted({0, *((k * per_pass // 128 - 2) * 128 for k in range(1, rows // per_pass + 1)), (rows - 1) // 128 * 128 - 256}):
        first = max(first, 0)
        yield first, min(rows, first + STEP)


def scale_range(fmt, cols, first, last):
    """Bytes of the scales of rows first .. last - 1, `first` a multiple of 128."""
    return slice(sparq.sparq_mx_scale_bytes(fmt, first, cols), sparq.sparq_mx_scale_bytes(fmt, last, cols))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", LARGE)
def test_codec(fmt, dtype, rows, cols):
    x = tensor(rows, rows, cols, dtype)
    m = x.float().abs().amax().view(1) if fmt == ref.NVFP4 else None
    codes, scales = buffers(fmt, rows, cols)
    sparq.sparq_quantize_mx(x, fmt, codes, scales, max_dev=m)
    out = torch.full_like(x, 7.0)
    sparq.sparq_dequantize_mx(codes, scales, fmt, out, max_dev=m)
    for first, last in pieces(rows, cols):
        c, s = buffers(fmt, last - first, cols)
        sparq.sparq_quantize_mx(x[first:last], fmt, c, s, max_dev=m)
        assert torch.equal(codes[first:last], c) and torch.equal(scales[scale_range(fmt, cols, first, last)], s)
        v = torch.empty_like(x[first:last])
        sparq.sparq_dequantize_mx(c, s, fmt, v, max_dev=m)
        assert torch.equal(out[first:last], v)
    # every element: near what it was, by its block's scale, by plain operations
    block = ref.BLOCK[fmt]
    pad = torch.nn.functional.pad(x.float(), (0, ref.up(cols, 32) - cols)).view(rows, -1, block)
    a = pad.abs().amax(-1, keepdim=True)
    far = (torch.nn.functional.pad(out.float(), (0, ref.up(cols, 32) - cols)).view(rows, -1, block) - pad).abs()
    # MXINT8: half a unit of 2^-6 (1 where 127.5 and above are clamped) of at most a; 4 bits: half of the largest step (2 of 6..8 units)
    # of at most a / 4 and what saturates (2 units), e4m3's half step (2^-4) or least scale beside it; bf16 rounds once more
    if fmt == ref.MXINT8:
        tol = a * 2.0 ** -6
    elif fmt == ref.MXFP4:
        tol = a * 0.5
    else:
        tol = a * (1 / 6 + 0.2) + m / 448 * 2.0 ** -9
    assert bool((far <= tol + 2.0 ** -8 * a).all())
    if fmt == ref.MXINT8:           # and its codes
        e = torch.where(a > 0, torch.frexp(a)[1] - 1, -127).clamp(min=-127)
        q = torch.round(torch.ldexp(pad.double(), 6 - e)).clamp(-127, 127)
        assert torch.equal(codes.view(pad.shape).double(), q)


def kept(rows, cols):
    codes, scales = buffers(ref.MXINT8, rows, cols)
    return codes, scales


def forward(x, up, y, act, c, s, uc=None, us=None):
    sparq.sparq_act_forward_mx8(x, act, y, c, s, up=up, up_codes=uc, up_scales=us)


@pytest.mark.parametrize("act", [sparq.ACT_RELU, sparq.ACT_GELU])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", LARGE)
def test_activations(act, gated, dtype, rows, cols):
    wide = tensor(cols, rows, cols * (2 if gated else 1), dtype)
    x, up = wide[:, :cols], wide[:, cols:] if gated else None
    k = [kept(rows, cols) for _ in range(2 if gated else 1)]
    y = torch.full((rows, cols), 7.0, dtype=dtype, device="cuda")
    forward(x, up, y, act, *k[0], *(k[1] if gated else ()))
    dy = tensor(3, rows, cols, dtype)
    d = torch.full_like(wide, 7.0)
    dx, dup = d[:, :cols], d[:, cols:] if gated else None
    sparq.sparq_act_backward_mx8(dy, *k[0], act, dx, **(dict(up_codes=k[1][0], up_scales=k[1][1], dup=dup) if gated else {}))
    sparq.sparq_check()
    for t, (c, s) in zip((x, up), k):
        c2, s2 = kept(rows, cols)
        sparq.sparq_quantize_mx(t, ref.MXINT8, c2, s2)          # tested above
        assert torch.equal(c, c2) and torch.equal(s, s2)
    for first, last in pieces(rows, cols):
        part = lambda t: t[first:last] if t is not None else None
        k2 = [kept(last - first, cols) for _ in k]
        y2 = torch.empty_like(y[first:last])
        forward(part(x), part(up), y2, act, *k2[0], *(k2[1] if gated else ()))
        assert torch.equal(y[first:last], y2)
        dx2, dup2 = torch.empty_like(y2), torch.empty_like(y2) if gated else None
        sparq.sparq_act_backward_mx8(dy[first:last], *k2[0], act, dx2, **(dict(up_codes=k2[1][0], up_scales=k2[1][1], dup=dup2) if gated else {}))
        assert torch.equal(dx[first:last], dx2) and (not gated or torch.equal(dup[first:last], dup2))
    if act == sparq.ACT_RELU:       # one rounding each: plain operations give the same bits
        want = torch.where(x > 0, x, 0.0).float()
        assert torch.equal(y, (want * up.float() if gated else want).to(dtype))
        values = [torch.empty((rows, cols), device="cuda") for _ in k]
        for v, (c, s) in zip(values, k):
            sparq.sparq_dequantize_mx(c, s, ref.MXINT8, v)
        on = values[0] > 0
        t = dy.float() * values[1] if gated else dy.float()
        assert torch.equal(dx, torch.where(on, t, t * 0.0).to(dtype))
        if gated:
            assert torch.equal(dup, (dy.float() * torch.where(on, values[0], 0.0)).to(dtype))


def beside(room, rows, cols, pitch, offset):
    return torch.as_strided(room, (rows, cols), (pitch, 1), offset)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (5, 15), (77, 17), (40, 33), (130, 100), (50, 201), (33, 1001), (9, 2500), (60001, 331)])
@pytest.mark.parametrize("place", ["x", "up", "plain"])
def test_forward_in_place(dtype, rows, cols, place):
    """y is x, y is up, y is x without a gate: as out of place, and nothing else is touched.  Vectors of such rows reach into others."""
    for offset, gap in ((0, 0), (1, 3)):
        pitch = 2 * cols + gap
        room = torch.full((offset + rows * pitch + 64,), 5.0, dtype=dtype, device="cuda")
        x, up = beside(room, rows, cols, pitch, offset), beside(room, rows, cols, pitch, offset + cols)
        x.copy_(tensor(cols, rows, cols, dtype))
        up.copy_(tensor(cols + 1, rows, cols, dtype))
        gate = place != "plain"
        k = [kept(rows, cols) for _ in range(4)]
        want = torch.empty((rows, cols), dtype=dtype, device="cuda")
        forward(x.contiguous(), up.contiguous() if gate else None, want, sparq.ACT_SILU, *k[0], *(k[1] if gate else ()))
        after = room.clone()
        y = up if place == "up" else x
        beside(after, rows, cols, pitch, y.storage_offset()).copy_(want)
        forward(x, up if gate else None, y, sparq.ACT_SILU, *k[2], *(k[3] if gate else ()))
        assert torch.equal(room, after)
        for a, b in zip(k[0] + (k[1] if gate else ()), k[2] + (k[3] if gate else ())):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (5, 15), (77, 17), (40, 33), (130, 100), (50, 201), (33, 1001), (9, 2500), (60001, 331)])
@pytest.mark.parametrize("place", ["dx", "dup", "plain"])
def test_backward_in_place(dtype, rows, cols, place):
    """dx is dy, dup is dy, dx is dy without a gate."""
    gate = place != "plain"
    k = [kept(rows, cols) for _ in range(2)]
    forward(tensor(1, rows, cols, dtype), tensor(2, rows, cols, dtype), torch.empty((rows, cols), dtype=dtype, device="cuda"), sparq.ACT_GELU, *k[0], *k[1])
    more = dict(up_codes=k[1][0], up_scales=k[1][1]) if gate else {}
    for offset, gap in ((0, 0), (1, 3)):
        pitch = 2 * cols + gap
        room = torch.full((offset + rows * pitch + 64,), 5.0, dtype=dtype, device="cuda")
        dx, dup = beside(room, rows, cols, pitch, offset), beside(room, rows, cols, pitch, offset + cols)
        dy = dup if place == "dup" else dx
        dy.copy_(tensor(3, rows, cols, dtype))
        want = torch.empty((rows, cols), dtype=dtype, device="cuda"), torch.empty((rows, cols), dtype=dtype, device="cuda")
        sparq.sparq_act_backward_mx8(dy.contiguous(), *k[0], sparq.ACT_GELU, want[0], **more, **(dict(dup=want[1]) if gate else {}))
        after = room.clone()
        beside(after, rows, cols, pitch, offset).copy_(want[0])
        if gate:
            beside(after, rows, cols, pitch, offset + cols).copy_(want[1])
        sparq.sparq_act_backward_mx8(dy, *k[0], sparq.ACT_GELU, dx, **more, **(dict(dup=dup) if gate else {}))
        assert torch.equal(room, after)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (300, 1000), (129, 333)])
def test_largest_magnitude_from_the_library(dtype, rows, cols):
    """NVFP4's m as sparq_absmax gathers it."""
    x = tensor(7, rows, cols, dtype).contiguous()
    m = torch.zeros(1, device="cuda")
    sparq.sparq_absmax(x, m)
    codes, scales = buffers(ref.NVFP4, rows, cols)
    sparq.sparq_quantize_mx(x, ref.NVFP4, codes, scales, max_dev=m)
    q, s = ref.quantize(x.float().cpu().numpy(), ref.NVFP4, float(x.float().abs().max()))
    assert torch.equal(codes.cpu(), torch.from_numpy(ref.pack(q, ref.NVFP4))) and torch.equal(scales.cpu(), torch.from_numpy(ref.lay_scales(s, ref.NVFP4)))
