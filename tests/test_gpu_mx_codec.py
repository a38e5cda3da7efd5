"""Quantization to the microscaled formats and back against the plain 64-bit implementation, bit for bit."""
import numpy as np
import pytest
import torch

import mx_reference as ref
import paper_2105_11010_b200 as sparq

pytestmark = pytest.mark.gpu

FORMATS = [ref.MXFP4, ref.NVFP4, ref.MXINT8]


def tensor(seed, rows, cols, dtype):
    rng = np.random.default_rng(seed)
    x = (rng.standard_normal((rows, cols)) * np.exp(rng.standard_normal((rows, 1)) * 3)).astype(np.float32)
    x[rng.random((rows, cols)) < 0.1] = 0.0
    return torch.from_numpy(x).to(dtype)


def buffers(fmt, rows, cols, fill=0xA5):
    n = ref.up(cols, 32)
    codes = torch.full((rows, n if fmt == 2 else n // 2), fill - 256 if fmt == 2 else fill, dtype=torch.int8 if fmt == 2 else torch.uint8, device="cuda")
    return codes, torch.full((sparq.sparq_mx_scale_bytes(fmt, rows, cols),), fill, dtype=torch.uint8, device="cuda")


def check(x, fmt, largest=None, xd=None):
    """Codes, scales (padding included) and decoded values of x in both types."""
    rows, cols = x.shape
    xd = x.cuda() if xd is None else xd
    codes, scales = buffers(fmt, rows, cols)
    m = torch.tensor([largest], dtype=torch.float32, device="cuda") if fmt == 1 else None
    sparq.sparq_quantize_mx(xd, fmt, codes, scales, max_dev=m)
    q, s = ref.quantize(x.float().numpy(), fmt, largest)
    assert np.array_equal(scales.cpu().numpy(), ref.lay_scales(s, fmt))
    assert np.array_equal(codes.cpu().numpy(), ref.pack(q, fmt))
    with np.errstate(invalid="ignore", over="ignore"):
        want = ref.values(q, s, fmt, cols).astype(np.float32)          # exact in fp32
        want = want * ref.tensor_scale(largest) if fmt == 1 else want
    for dt in (torch.float32, torch.bfloat16):
        out = torch.full((rows, cols + 3), 7.0, dtype=dt, device="cuda")
        for view in (out[:, :cols], torch.empty((rows, cols), dtype=dt, device="cuda")):
            sparq.sparq_dequantize_mx(codes, scales, fmt, view, max_dev=m)
            assert torch.equal(torch.nan_to_num(view.float().cpu(), 1e30), torch.nan_to_num(torch.from_numpy(want).to(dt).float(), 1e30))
        assert bool((out[:, cols:] == 7.0).all())                     # between the rows
    sparq.sparq_check()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 15), (1, 16), (1, 17), (2, 31), (3, 32), (5, 33), (127, 64), (128, 65), (129, 200), (260, 520)])
def test_codes_scales_and_values(fmt, dtype, rows, cols):
    x = tensor(rows * 1000 + cols, rows, cols, dtype)
    check(x, fmt, float(x.abs().max()))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("pitch,offset", [(200, 0), (201, 0), (208, 1), (208, 8), (216, 4)])
def test_strides_and_alignments(fmt, pitch, offset):
    for dtype in (torch.float32, torch.bfloat16):
        x = tensor(7, 40, 200, dtype)
        room = torch.zeros(40 * pitch + 64, dtype=dtype, device="cuda")
        view = room[offset:offset + 40 * pitch].view(40, pitch)[:, :200]
        view.copy_(x)
        check(x, fmt, float(x.abs().max()), view)


@pytest.mark.parametrize("fmt", FORMATS)
def test_every_tie_and_border(fmt):
    """Halfway points, the largest element of a block just below a power of two, signed zeros."""
    halves = np.array([0, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, 6, 7, 7.9999995], np.float32)
    near = np.concatenate([halves, np.nextafter(halves, np.float32(0)), np.nextafter(halves, np.float32(9))])
    v = np.concatenate([near, -near, (np.arange(255) - 127).astype(np.float32) / 64 + np.float32(1 / 128), [-0.0]]).astype(np.float32)
    rows = []
    for top in (4.0, 6.0, 7.9999995, 1.0, 1.9999999, 2.0):
        b = np.zeros((ref.up(len(v), 15) // 15, 16), np.float32)
        b[:, 1:].flat[:len(v)] = np.clip(v, -top, top)
        b[:, 0] = top
        rows.append(b)
    x = torch.from_numpy(np.concatenate(rows))
    for scale in (1.0, 2.0 ** -30, 2.0 ** 40):
        check((x * scale).reshape(-1, 16), fmt, 8.0 * scale)


@pytest.mark.parametrize("fmt", FORMATS)
def test_zeros_subnormals_and_the_ends_of_the_range(fmt):
    x = torch.zeros((7, 96))
    x[1, :] = 1e-45
    x[2, 3] = -2.0 ** -126
    x[3, 40] = 2.0 ** -149
    x[4, :] = torch.finfo(torch.float32).max
    x[5, 0], x[5, 33], x[5, 70] = 1e38, 1e-38, -3e38
    x[6, 95] = 2.0 ** 127
    check(x, fmt, float(x.abs().max()))
    check(x[:4], fmt, float(x[:4].abs().max()))
    check(x[:1], fmt, 0.0)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_block_with_a_number_that_is_none(fmt, bad):
    x = tensor(3, 5, 130, torch.float32)
    x[1, 50] = bad
    x[4, 129] = bad
    check(x, fmt, 9.0)


def test_a_largest_magnitude_that_does_not_fit():
    """Static statistics: values beyond them saturate; infinities and NaN as the statistic read as NaN or as they are defined."""
    x = tensor(5, 9, 64, torch.float32)
    for largest in (1e-3, 1e6, 2.0 ** -120, float("nan"), float("inf")):
        check(x, ref.NVFP4, largest)


def test_rows_beyond_32_bits_of_offset():
    """A row pitch so long that element offsets pass 2^32; the rows between are not touched."""
    pitch = 1 << 31
    room = torch.empty(2 * pitch + 64, dtype=torch.bfloat16, device="cuda")
    view = torch.as_strided(room, (3, 64), (pitch, 1))
    x = tensor(2, 3, 64, torch.bfloat16)
    view.copy_(x)
    check(x, ref.MXFP4, None, view)
    codes, scales = buffers(2, 3, 64)
    sparq.sparq_quantize_mx(view, 2, codes, scales)
    view.zero_()
    sparq.sparq_dequantize_mx(codes, scales, 2, view)
    q, s = ref.quantize(x.float().numpy(), 2)
    assert np.array_equal(view.float().cpu().numpy(), ref.values(q, s, 2, 64).astype(np.float32))


def test_nothing_is_a_no_op():
    codes, scales = buffers(0, 4, 64)
    before = codes.clone(), scales.clone()
    sparq.sparq_quantize_mx(torch.empty((0, 64), device="cuda"), 0, codes, scales)
    sparq.sparq_quantize_mx(torch.empty((4, 0), device="cuda"), 0, codes, scales)
    assert torch.equal(codes, before[0]) and torch.equal(scales, before[1])


def test_small_buffers_are_refused():
    x = torch.zeros((4, 64), device="cuda")
    codes, scales = buffers(0, 4, 64)
    for c, s in ((codes[:3], scales), (codes, scales[:-1]), (codes.view(torch.int8), scales), (codes.t(), scales)):
        with pytest.raises(ValueError):
            sparq.sparq_quantize_mx(x, 0, c, s)
    with pytest.raises(ValueError):
        sparq.sparq_quantize_mx(x.t(), 0, codes, scales)
    with pytest.raises(ValueError):
        sparq.sparq_quantize_mx(x.half(), 0, codes, scales)
