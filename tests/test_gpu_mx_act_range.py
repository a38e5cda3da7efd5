"""Activation functions of fp32 tensors over the whole range of their logistic factor: few units of the last place, also where it leaves the
range of fp32 and the result does not.

Tolerance, in units U = 2^-23 of a value.  With h = exp(-|z| / 2) off by 2.5 (the approximate power of two 2, half of one where its correction is
added), its square t is off by 5.5 and r = 1 / (1 + t) by 1 + 0.5 + 5.5 t / (1 + t) <= 4.25.  s(z) x is x h h r or x r, with three products:
5 + 4.25 + 1.5 < 11 units, and two roundings of subnormals, 2^-148.  The derivative s + c z' s (1 - s) is h (h (q + r)) or t q + r with
q = c z' r^2 off by 8.5 + 4.5 (z' and three products): 13 for q, 5.5 for t or h h, 1.5 for the sum and two products, 20 units of
|s| + |c z' s (1 - s)|.  GELU's argument z in fp32 has two rounded
constants and four roundings, 3 units: the logistic function changes by (1 - s) |z| 3 units, the derivative's terms by as much of theirs."""
import numpy as np
import pytest
import torch

import mx_reference as ref
import paper_2105_11010_b200 as sparq

pytestmark = pytest.mark.gpu

ACTS = [sparq.ACT_SILU, sparq.ACT_GELU]
U = 2.0 ** -23
LAST = 2.0 ** -148


def forward(x, act):
    rows, cols = x.shape
    y = torch.empty_like(x)
    codes = torch.empty((rows, ref.up(cols, 32)), dtype=torch.int8, device="cuda")
    scales = torch.empty((rows, ref.up(ref.up(cols, 32) // 32, 16)), dtype=torch.uint8, device="cuda")
    sparq.sparq_act_forward_mx8(x, act, y, codes, scales)
    return y.float().cpu().numpy().astype(np.float64), codes, scales


def values(act):
    """Every size of the result, steps between the borders, and ends of the range."""
    far = 130.0 if act == sparq.ACT_SILU else 12.0
    x = np.concatenate([np.linspace(-far, far, 64 * 509), np.linspace(-far, -0.6 * far, 64 * 101), 2.0 ** -np.arange(0.0, 149.0, 0.5),
                        -(2.0 ** -np.arange(0.0, 149.0, 0.5)), [0.0, -0.0, 1e30, -1e30, 3e38, -3e38]]).astype(np.float32)
    return np.concatenate([x, np.zeros(-len(x) % 64, np.float32)]).reshape(-1, 64)


@pytest.mark.parametrize("act", ACTS)
def test_function(act):
    x = values(act)
    got, _, _ = forward(torch.from_numpy(x).cuda(), act)
    with np.errstate(over="ignore"):
        y, _, z, s = ref.act(x, act)
    units = 11 + (3 * np.abs(np.maximum(z, -1e6)) * (1 - s) if act == sparq.ACT_GELU else 0)
    assert (np.abs(got - y) <= units * U * np.abs(y) + LAST).all()


@pytest.mark.parametrize("act", ACTS)
def test_derivative(act):
    """Kept values that 8 bits hold exactly: whole numbers up to 127 (quarters up to 15 for GELU)."""
    unit = 1.0 if act == sparq.ACT_SILU else 0.125
    x = (np.arange(-127, 129) % 128 * np.sign(np.arange(-127, 129))).astype(np.float32).reshape(8, 32)
    x[:, 0] = 127.0
    x = np.concatenate([x, -x]) * np.float32(unit)
    t = torch.from_numpy(x).cuda()
    _, codes, scales = forward(t, act)
    dx = torch.empty_like(t)
    sparq.sparq_act_backward_mx8(torch.ones_like(t), codes, scales, act, dx)
    got = dx.cpu().numpy().astype(np.float64)
    x = x.astype(np.float64)
    _, d, z, s = ref.act(x, act)
    g = np.sqrt(8 / np.pi)
    dz = np.ones_like(x) if act == sparq.ACT_SILU else g * (1 + 3 * 0.044715 * x ** 2)
    n = 1 / (1 + np.exp(z))
    second = np.abs(x * dz) * s * n
    tol = 20 * U * (s + second) + LAST
    if act == sparq.ACT_GELU:
        tol = tol + 3 * np.abs(z) * U * (s * n + second)
    assert (np.abs(got - d) <= tol).all()


@pytest.mark.parametrize("act", ACTS)
def test_bf16(act):
    """2^-14 from the approximate power of two and from z, half a step of bf16 (2^-8 of the value), 2^-119 where the factor is below 2^-126."""
    x = torch.from_numpy(values(act)).cuda().bfloat16()
    got, _, _ = forward(x, act)
    with np.errstate(over="ignore"):
        y = ref.act(x.float().cpu().numpy(), act)[0]
    assert (np.abs(got - y) <= (2.0 ** -8 + 2.0 ** -14) * np.abs(y) * (1 + 2.0 ** -8) + 2.0 ** -119).all()


@pytest.mark.parametrize("act", ACTS)
def test_infinities_and_nan(act):
    x = torch.tensor([[float("inf"), -float("inf"), float("nan")] + [1.0] * 29], device="cuda")
    got, _, _ = forward(x, act)
    assert got[0, 0] == np.inf and np.isnan(got[0, 1]) and np.isnan(got[0, 2])          # x / (1 + exp(-x)) at -inf: inf / inf
