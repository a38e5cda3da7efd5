"""Activation functions that keep their inputs in 8 bits, and their backward pass, against the formulas in 64 bits.

Tolerance.  The kernels work in fp32 with the approximate power of two (exp(-z) off by 2 + |1.16 z| units of 2^-23, the multiplication by log2 e
included) and reciprocal (1 unit).  With E that error of exp(-z) and z itself off by 4 roundings (4 |z| 2^-24), s(z) = 1 / (1 + exp(-z)) is off by s (1 - s) (E + 2 |z| 2^-23) + 3 s 2^-23,
written as s e; products add 2^-24 each.  The derivative s + c s (1 - s) z' is off by s e, |c z'| times the errors of s (1 - s), and
five roundings of the second term.  bf16 outputs add half a step, 2^-8 of the result."""
import numpy as np
import pytest
import torch

import mx_reference as ref
import paper_2105_11010_b200 as sparq

pytestmark = pytest.mark.gpu

ACTS = [sparq.ACT_IDENTITY, sparq.ACT_RELU, sparq.ACT_SILU, sparq.ACT_GELU]
U = 2.0 ** -23


def bounds(x, kind):
    """(act, act', error of act, error of act') in 64 bits."""
    y, d, z, s = ref.act(x, kind)
    if kind < 2:
        return y, d, 0 * y, 0 * d
    e = ((2 + 1.16 * np.abs(z) + 2 * np.abs(z)) * (1 - s) + 3) * U
    big = np.abs(x) > (60 if kind == 3 else 120)
    dz = np.ones_like(x) if kind == 2 else np.sqrt(8 / np.pi) * (1 + 3 * 0.044715 * np.minimum(np.abs(x), 64) ** 2)
    c = np.minimum(np.abs(x), 64 if kind == 3 else 128)
    second = c * dz * (s * e * (1 - s) + s * (s * e + U / 2)) + 5 * U / 2 * c * dz * s * (1 - s)
    ed = s * e + np.where(big, 1e-30, second) + U / 2 * np.abs(d)
    return y, d, np.abs(y) * (e + U / 2) + 1e-36 * np.abs(x), ed + 1e-36


def pieces(seed, rows, cols, gated, dtype):
    rng = np.random.default_rng(seed)
    wide = (rng.standard_normal((rows, cols * (2 if gated else 1))) * 3).astype(np.float32)
    wide[rng.random(wide.shape) < 0.05] *= 20
    t = torch.from_numpy(wide).to(dtype).cuda()
    return t[:, :cols], t[:, cols:] if gated else None


def kept(rows, cols):
    return (torch.full((rows, ref.up(cols, 32)), 85, dtype=torch.int8, device="cuda"),
            torch.full((rows, ref.up(ref.up(cols, 32) // 32, 16)), 85, dtype=torch.uint8, device="cuda"))


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 17), (5, 32), (7, 100), (64, 513), (130, 1024)])
def test_forward_and_backward(act, gated, dtype, rows, cols):
    x, up = pieces(rows + cols, rows, cols, gated, dtype)
    y = torch.empty((rows, cols), dtype=dtype, device="cuda")
    (c, s), (uc, us) = kept(rows, cols), kept(rows, cols) if gated else (None, None)
    sparq.sparq_act_forward_mx8(x, act, y, c, s, up=up, up_codes=uc, up_scales=us)
    v, _, ev, _ = bounds(f64(x), act)
    tol = ev
    if gated:
        u = f64(up)
        v, tol = v * u, ev * np.abs(u) + U / 2 * np.abs(v * u)
    assert (np.abs(f64(y) - v) <= tol + half_step(dtype) * (np.abs(v) + tol)).all()
    back = []
    for t, codes, scales in ((x, c, s), (up, uc, us)):
        if t is None:
            continue
        q, e = ref.quantize(t.float().cpu().numpy(), ref.MXINT8)
        assert np.array_equal(codes.cpu().numpy(), q.astype(np.int8))
        assert np.array_equal(scales.flatten().cpu().numpy(), ref.lay_scales(e, ref.MXINT8))
        back.append(ref.values(q, e, ref.MXINT8, cols))

    rng = np.random.default_rng(1)
    dy = torch.from_numpy((rng.standard_normal((rows, cols)) * 1e-2).astype(np.float32)).to(dtype).cuda()
    dx = torch.empty((rows, cols), dtype=dtype, device="cuda")
    dup = torch.empty_like(dx) if gated else None
    sparq.sparq_act_backward_mx8(dy, c, s, act, dx, up_codes=uc, up_scales=us, dup=dup)
    sparq.sparq_check()
    g = f64(dy)
    v, d, ev, ed = bounds(back[0], act)
    t = g * back[1] if gated else g
    want = t * d
    tol = np.abs(t) * ed + U * np.abs(want) + 1e-40
    assert (np.abs(f64(dx) - want) <= tol + half_step(dtype) * (np.abs(want) + tol)).all()
    if gated:
        want = g * v
        tol = np.abs(g) * ev + U / 2 * np.abs(want) + 1e-40
        assert (np.abs(f64(dup) - want) <= tol + half_step(dtype) * (np.abs(want) + tol)).all()


@pytest.mark.parametrize("act", [sparq.ACT_SILU, sparq.ACT_GELU])
def test_gradient_against_differences(act):
    """dx from the kernel against central differences of the kernel's own forward pass, at inputs that 8 bits hold exactly.

    With step h = 2^-7 the difference quotient is off by h^2 / 6 |act'''| (at most 1 for either function on this range, so below
    1.1e-5) and by the forward pass's rounding over h, both sides: 2 * 12 * 2^-23 * |y| / (2 h)."""
    h = 2.0 ** -7
    x = (np.arange(64 * 32).reshape(64, 32) % 127 - 63).astype(np.float32) / 16           # multiples of 2^-4 up to 4
    x[:, 0] = 4.0
    t = torch.from_numpy(x).cuda()
    (c, s), dx = kept(64, 32), torch.empty((64, 32), device="cuda")
    ys = []
    for d in (h, -h):
        ys.append(torch.empty_like(t))
        sparq.sparq_act_forward_mx8(t + d, act, ys[-1], c, s)
    sparq.sparq_act_forward_mx8(t, act, torch.empty_like(t), c, s)
    sparq.sparq_act_backward_mx8(torch.ones_like(t), c, s, act, dx)
    want = (f64(ys[0]) - f64(ys[1])) / (2 * h)
    assert np.abs(f64(dx) - want).max() <= h * h / 6 + 12 * U * 4.1 / h + 1e-6


@pytest.mark.parametrize("act", [sparq.ACT_RELU, sparq.ACT_SILU, sparq.ACT_GELU])
def test_far_values(act):
    """Inputs so large that squares and cubes overflow: the functions' limits, and no NaN."""
    x = torch.tensor([[3e38, -3e38, 1e20, -1e20, 200.0, -200.0, 1e4, -1e4] * 4 + [0.0, -0.0, 1e-40, -1e-40] * 8], device="cuda")
    y, dx, (c, s) = torch.empty_like(x), torch.empty_like(x), kept(1, 64)
    sparq.sparq_act_forward_mx8(x, act, y, c, s)
    assert torch.equal(y[0, :32], torch.where(x[0, :32] > 0, x[0, :32], 0.0))
    for v in (3e38, 1e20, 200.0):
        t = torch.full_like(x, v)
        t[0, ::2] *= -1
        sparq.sparq_act_forward_mx8(t, act, y, c, s)
        sparq.sparq_act_backward_mx8(torch.ones_like(x), c, s, act, dx)
        assert torch.equal(dx, (t > 0).float())


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("gated", [False, True])
def test_numbers_that_are_none_stay_in_their_blocks(act, gated):
    x, up = pieces(5, 4, 96, gated, torch.float32)
    x = x.clone()
    x[1, 40] = float("nan")
    x[2, 0] = float("inf")
    up = up.clone() if gated else None
    if gated:
        up[3, 95] = -float("inf")
    y, dy, dx = torch.empty_like(x), torch.ones_like(x), torch.empty_like(x)
    (c, s), (uc, us) = kept(4, 96), kept(4, 96) if gated else (None, None)
    dup = torch.empty_like(x) if gated else None
    sparq.sparq_act_forward_mx8(x, act, y, c, s, up=up, up_codes=uc, up_scales=us)
    sparq.sparq_act_backward_mx8(dy, c, s, act, dx, up_codes=uc, up_scales=us, dup=dup)
    nan = np.zeros((4, 96), bool)
    nan[1, 32:64] = nan[2, :32] = True
    if gated:
        assert np.array_equal(torch.isnan(dup).cpu().numpy(), nan)
        nan[3, 64:] = True
    assert np.array_equal(torch.isnan(dx).cpu().numpy(), nan)


def test_in_place_and_strided():
    x, up = pieces(9, 50, 200, True, torch.bfloat16)
    y = torch.empty((50, 200), dtype=torch.bfloat16, device="cuda")
    (c, s), (uc, us) = kept(50, 200), kept(50, 200)
    sparq.sparq_act_forward_mx8(x, sparq.ACT_SILU, y, c, s, up=up, up_codes=uc, up_scales=us)
    both = torch.cat([x, up], 1)
    a, b = both[:, :200], both[:, 200:]
    (c2, s2), (uc2, us2) = kept(50, 200), kept(50, 200)
    sparq.sparq_act_forward_mx8(a, sparq.ACT_SILU, a, c2, s2, up=b, up_codes=uc2, up_scales=us2)
    assert torch.equal(a, y) and torch.equal(b, up) and torch.equal(c, c2) and torch.equal(uc, uc2) and torch.equal(s, s2)
    dy = torch.randn((50, 200), device="cuda").bfloat16()
    dx, dup = torch.empty_like(dy), torch.empty_like(dy)
    sparq.sparq_act_backward_mx8(dy, c, s, sparq.ACT_SILU, dx, up_codes=uc, up_scales=us, dup=dup)
    wide = torch.full((50, 407), 3.0, dtype=torch.bfloat16, device="cuda")
    sparq.sparq_act_backward_mx8(dy, c, s, sparq.ACT_SILU, wide[:, 1:201], up_codes=uc, up_scales=us, dup=wide[:, 203:403])
    assert torch.equal(wide[:, 1:201], dx) and torch.equal(wide[:, 203:403], dup)
    assert bool((wide[:, [0, 201, 202, 403, 406]] == 3.0).all())
    sparq.sparq_act_backward_mx8(dy, c, s, sparq.ACT_SILU, dy, up_codes=uc, up_scales=us, dup=dup)
    assert torch.equal(dy, dx)


def test_partners_of_another_shape_are_refused():
    x = torch.zeros((4, 64), device="cuda")
    c, s = kept(4, 64)
    for y, kw in ((x[:3], {}), (x[:, :32], {}), (x.bfloat16(), {}), (x, dict(up=torch.zeros((4, 66), device="cuda")[:, :64], up_codes=c, up_scales=s))):
        with pytest.raises(ValueError):
            sparq.sparq_act_forward_mx8(x, 2, y, c, s, **kw)
    with pytest.raises(sparq.SparqError):
        sparq.sparq_act_forward_mx8(x, 2, x, c, s, up=x)
