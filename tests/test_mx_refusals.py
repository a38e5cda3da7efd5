"""Microscaled formats: sizes, and the calls that are refused, on the host."""
import ctypes

import pytest
import torch

import mx_reference as ref
import paper_2105_11010_b200 as sparq
from paper_2105_11010_b200._binding import _CMxEpilogue

P = 1 << 20          # a pointer that is never read: the call is refused before it touches a device


@pytest.mark.parametrize("fmt", [0, 1, 2])
@pytest.mark.parametrize("rows,cols", [(0, 0), (1, 1), (1, 32), (128, 64), (129, 65), (3, 513), (1000, 4097)])
def test_sizes(fmt, rows, cols):
    n = ref.up(cols, 32)
    scales = n // ref.BLOCK[fmt]
    assert sparq.sparq_mx_code_bytes(fmt, rows, cols) == rows * (n if fmt == 2 else n // 2)
    assert sparq.sparq_mx_scale_bytes(fmt, rows, cols) == (rows * ref.up(scales, 16) if fmt == 2 else ref.up(rows, 128) * ref.up(scales, 4))


def test_sizes_refuse():
    for f in (sparq.sparq_mx_code_bytes, sparq.sparq_mx_scale_bytes):
        for args, code in (((3, 1, 1), -1), ((-1, 1, 1), -1), ((0, -1, 1), -1), ((0, 1, -1), -1), ((0, 1 << 41, 1), -2), ((0, 1, (1 << 31) - 255), -2), ((0, (1 << 31) - 257, (1 << 31) - 257), -2)):
            with pytest.raises(sparq.SparqError) as e:
                f(*args)
            assert e.value.code == code, args


def refused(code, word, rc):
    assert rc == code and word in sparq.sparq_last_error(), (rc, sparq.sparq_last_error())


@pytest.mark.parametrize("quantize", [True, False])
def test_codec(quantize):
    L = sparq.load_library()

    def call(x=P, dtype=0, rows=4, cols=64, ld=64, fmt=0, mx=None, codes=P, scales=P):
        if quantize:
            return L.sparq_quantize_mx(x, dtype, rows, cols, ld, fmt, mx, codes, scales, None)
        return L.sparq_dequantize_mx(codes, scales, rows, cols, fmt, mx, x, dtype, ld, None)
    refused(-1, "format", call(fmt=3))
    refused(-1, "max_dev", call(fmt=1))
    refused(-1, "max_dev", call(mx=P))
    refused(-2, "max_dev", call(fmt=1, mx=P + 2))
    refused(-1, "dtype", call(dtype=2))
    refused(-1, "negative", call(rows=-1))
    refused(-1, "NULL", call(x=None))
    refused(-1, "NULL", call(codes=None))
    refused(-1, "NULL", call(scales=None))
    refused(-1, "leading dimension", call(ld=63))
    refused(-2, "aligned", call(x=P + 2))
    refused(-2, "aligned", call(dtype=1, x=P + 1))
    refused(-2, "aligned", call(codes=P + 8))
    refused(-2, "aligned", call(scales=P + 4))
    refused(-2, "2^31", call(rows=1 << 41))
    refused(-2, "more than any device", call(rows=1 << 30, ld=1 << 35))
    assert call(rows=0, x=None, codes=None, scales=None) == 0 and call(cols=0, ld=0, x=None, codes=None, scales=None) == 0


def test_gemm():
    L = sparq.load_library()

    def call(A=P, As=P, B=P, Bs=P, M=4, N=4, K=64, fmt=0, e=None, **epi):
        e = _CMxEpilogue(**{"f32_out": P, **epi}) if e is None else e
        return L.sparq_gemm_mxf4(A, As, B, Bs, M, N, K, fmt, ctypes.byref(e) if e else None, None)
    refused(-1, "format", call(fmt=2))
    refused(-1, "epilogue", call(e=False))
    refused(-1, "a_max", call(fmt=1, b_max=P))
    refused(-1, "b_max", call(fmt=1, a_max=P))
    refused(-1, "a_max", call(a_max=P))
    refused(-1, "no output", call(f32_out=None))
    refused(-1, "negative", call(M=-1))
    refused(-1, "K is 0", call(K=0))
    refused(-1, "NULL", call(Bs=None))
    refused(-2, "2^31", call(N=(1 << 31) - 256))
    refused(-2, "2^31", call(K=1 << 40))
    for name in ("A", "As", "B", "Bs"):
        refused(-2, "aligned", call(**{name: P + 8}))
    refused(-2, "aligned", call(f32_out=P + 2))
    refused(-2, "aligned", call(bf16_out=P + 1))
    refused(-2, "aligned", call(bias=P + 1))
    assert call(M=0, A=None) == 0 and call(N=0, B=None) == 0


@pytest.mark.parametrize("forward", [True, False])
def test_act(forward):
    L = sparq.load_library()

    def call(x=P, dtype=0, rows=4, cols=64, ld=64, act=2, y=P, ldy=64, codes=P, scales=P, up=None, uc=None, us=None):
        if forward:
            return L.sparq_act_forward_mx8(x, up, dtype, rows, cols, ld, act, y, ldy, codes, scales, uc, us, None)
        return L.sparq_act_backward_mx8(x, dtype, rows, cols, ld, act, codes, scales, uc, us, y, up, ldy, None)
    refused(-1, "dtype", call(dtype=5))
    refused(-1, "act", call(act=4))
    refused(-1, "act", call(act=-1))
    refused(-1, "negative", call(cols=-1))
    for name in ("x", "y", "codes", "scales"):
        refused(-1, "NULL", call(**{name: None}))
    for names in ({"up": P}, {"uc": P}, {"us": P}, {"up": P, "uc": P}, {"uc": P, "us": P}):
        refused(-1, "together", call(**names))
    refused(-1, "leading dimension", call(ld=60))
    refused(-1, "leading dimension", call(ldy=60))
    refused(-2, "aligned", call(x=P + 1))
    refused(-2, "aligned", call(y=P + 2))
    refused(-2, "aligned", call(codes=P + 8))
    refused(-2, "aligned", call(up=P, uc=P, us=P + 1))
    refused(-2, "2^31", call(rows=1 << 41))
    refused(-1, "in place", call(ldy=72))
    refused(-1, "in place", call(ld=72))
    if forward:
        refused(-1, "in place", call(up=P + 4096, uc=P, us=P, y=P + 4096, ld=72))
    else:
        refused(-1, "in place", call(up=P, uc=P, us=P, y=P + 4096, ld=72))
        refused(-1, "one matrix", call(x=P + 8192, up=P, uc=P, us=P))
    assert call(rows=0, x=None) == 0 and call(cols=0, x=None) == 0


def test_wgrad():
    L = sparq.load_library()

    def call(dy=P, ld=64, codes=P, scales=P, M=4, N=64, K=64, acc=0, dw=P):
        return L.sparq_wgrad_mx8(dy, ld, codes, scales, M, N, K, acc, dw, None, 0, None)
    refused(-1, "negative", call(K=-1))
    refused(-1, "dw", call(dw=None))
    refused(-2, "aligned", call(dw=P + 2))
    refused(-2, "2^31", call(M=1 << 31))
    for name in ("dy", "codes", "scales"):
        refused(-1, "NULL", call(**{name: None}))
    refused(-1, "leading dimension", call(ld=56))
    refused(-2, "multiple of 8", call(M=1, ld=5, dy=P + 8))
    refused(-2, "multiple of 8", call(ld=68))
    refused(-2, "multiple of 8", call(dy=P + 8))
    refused(-2, "aligned", call(codes=P + 4))
    refused(-1, "negative", L.sparq_wgrad_mx8_workspace_bytes(4, -1, 4))
    refused(-2, "2^31", L.sparq_wgrad_mx8_workspace_bytes(4, 1 << 31, 4))
    assert L.sparq_wgrad_mx8_workspace_bytes(0, 4, 4) == 0
    assert call(N=0, dw=None) == 0 and call(K=0, dw=None) == 0 and call(M=0, acc=1, dy=None) == 0


def test_tensors():
    """The call module: host tensors, wrong types, sizes and strides."""
    x, c, s = torch.zeros((4, 64)), torch.zeros((4, 32), dtype=torch.uint8), torch.zeros(512, dtype=torch.uint8)
    for f in (lambda: sparq.sparq_quantize_mx(x, 0, c, s), lambda: sparq.sparq_dequantize_mx(c, s, 0, x),
              lambda: sparq.sparq_gemm_mxf4(c, s, c, s, 0, f32_out=torch.zeros((4, 4))),
              lambda: sparq.sparq_act_forward_mx8(x, 1, x, c, s), lambda: sparq.sparq_act_backward_mx8(x, c, s, 1, x),
              lambda: sparq.sparq_wgrad_mx8(x, c, s, x)):
        with pytest.raises(ValueError):
            f()
    with pytest.raises(TypeError):
        sparq.sparq_quantize_mx(None, 0, c, s)
