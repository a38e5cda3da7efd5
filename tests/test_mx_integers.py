"""Integers of the microscaled calls that do not fit the C ABI's: refused, not cut off to others that are valid."""
import pytest
import torch

import paper_2105_11010_b200 as sparq

WRAPS = [1 << 32, (1 << 32) + 1, -(1 << 32), (1 << 32) + 2]


@pytest.mark.parametrize("fmt", WRAPS)
def test_sizes(fmt):
    for f in (sparq.sparq_mx_code_bytes, sparq.sparq_mx_scale_bytes):
        with pytest.raises(ValueError, match="fmt does not fit 32 bits"):
            f(fmt, 4, 64)
        with pytest.raises(ValueError, match="rows does not fit 64 bits"):
            f(0, 1 << 64, 64)
        with pytest.raises(ValueError, match="cols does not fit 64 bits"):
            f(0, 4, (1 << 64) + 64)
    with pytest.raises(ValueError, match="M does not fit 64 bits"):
        sparq.sparq_wgrad_mx8_workspace_bytes(1 << 64, 4, 4)


@pytest.mark.parametrize("value", WRAPS)
def test_formats_and_functions(value):
    x, c, s = torch.zeros((4, 64)), torch.zeros((4, 32), dtype=torch.uint8), torch.zeros(512, dtype=torch.uint8)
    for f in (lambda: sparq.sparq_quantize_mx(x, value, c, s), lambda: sparq.sparq_dequantize_mx(c, s, value, x),
              lambda: sparq.sparq_gemm_mxf4(c, s, c, s, value, f32_out=torch.zeros((4, 4)))):
        with pytest.raises(ValueError, match="fmt does not fit 32 bits"):
            f()
    for f in (lambda: sparq.sparq_act_forward_mx8(x, value, x, c, s), lambda: sparq.sparq_act_backward_mx8(x, c, s, value, x)):
        with pytest.raises(ValueError, match="act does not fit 32 bits"):
            f()
