"""Activation functions of sparq_linear by their relative error, over the range where they have any, in every form of launch."""
import pytest
import torch

import paper_2105_11010_b200 as sparq
from ffn_reference import F64, HALVES, inside
from test_gpu_linear import room

pytestmark = pytest.mark.gpu


def exactly(z, act):
    """x s(t) with s(t) = exp(t) / (1 + exp(t)), in 64 bits without the loss of a difference near the function's tail."""
    t = z if act == 2 else 2.0 * (2.0 / torch.pi) ** 0.5 * (z + 0.044715 * z ** 3)
    e = torch.exp(-t.abs())
    return z * torch.where(t < 0, e, torch.ones_like(e)) / (1.0 + e)


def allowed(y, out_type):
    """The functions' own relative error (2^-14 beside 16 bits, a few units of 2^-23 beside 32) and half a step of the output's rounding: relative, or of the smallest
    steps; results below 2^-119 may be 0 beside 16 bits."""
    own, least = {torch.float32: (8 * 2.0 ** -23, 2.0 ** -146), torch.bfloat16: (2.0 ** -14, 2.0 ** -119), torch.float16: (2.0 ** -14, 2.0 ** -25)}[out_type]
    return y.abs() * (own + torch.finfo(out_type).eps / 2 * (1 + own)) + least


@pytest.mark.parametrize("act", [2, 3])
@pytest.mark.parametrize("half,out_type", [("bf16", None), ("f16", None), ("bf16", torch.float32), ("f16", torch.float32)])
@pytest.mark.parametrize("rows,n", [(3, 136), (40, 4104), (200, 1000), (2300, 4104)])
def test_relative_error(rows, n, half, out_type, act):
    """z[i][j] = a[i] + b[j], sums of two numbers of 16 bits each that fp32 holds: rows of neighbours far apart, rows of neighbours close together, and values on either side of those where
    the function is taken another way (-43 for silu, -7.5 for gelu)."""
    dt = HALVES[half]
    ot = out_type or dt
    low, high, edge = (-100.0, 40.0, -43.0) if act == 2 else (-14.0, 9.0, -7.5)
    for spread in (0.0, 0.25, 20.0 if act == 2 else 4.0):
        a = torch.linspace(low, high, rows)
        a[::3] = edge
        x, w = torch.zeros((rows, 16), dtype=dt, device="cuda"), torch.zeros((n, 16), dtype=dt, device="cuda")
        steps = 4.0 if act == 2 else 32.0           # (multiples of a quarter, or of 2^-5: whole sums)
        x[:, 0], x[:, 1], w[:, 0] = (torch.round(a * steps) / steps).to(dt).cuda(), 1.0, 1.0
        w[:, 1] = torch.linspace(-spread, spread, n).to(dt).cuda()
        z = x[:, :1].to(F64) + w[:, 1].to(F64)
        exact = z.to(torch.float32).to(F64) == z
        assert exact.float().mean() > 0.5
        out = room(rows, n, ot)
        sparq.sparq_linear(x, w, out, act=act)
        y = exactly(z, act)
        inside(torch.where(exact, out.to(F64), y), y, allowed(y, ot))
    sparq.sparq_check()
