"""Weight gradients from inputs kept in 8 bits against 64-bit sums.

Tolerance.  Products of a bf16 value and a kept value are exact in the tensor cores' fp32.  Every output sees at most 16 additions
within each step of 16 tokens and one per step, each off by less than a unit 2^-23 of the largest partial sum, which
sum |dy x| bounds.  The kernel restarts the sum every 512 tokens (32 steps) and adds the parts, rounded to nearest:
(16 + 32 + M / 512 + 8) 2^-23 sum |dy x|, the 8 for a split reduction and the accumulation into dw."""
import numpy as np
import pytest
import torch

import mx_reference as ref
import paper_2105_11010_b200 as sparq

pytestmark = pytest.mark.gpu


def kept(x):
    """(codes, scales, 64-bit values) of a device matrix, by the library's own quantization (tested by itself)."""
    rows, cols = x.shape
    c = torch.empty((rows, ref.up(cols, 32)), dtype=torch.int8, device="cuda")
    s = torch.empty((rows, ref.up(ref.up(cols, 32) // 32, 16)), dtype=torch.uint8, device="cuda")
    sparq.sparq_quantize_mx(x, sparq.FORMAT_MXINT8, c, s)
    v = torch.empty((rows, cols), device="cuda")
    sparq.sparq_dequantize_mx(c, s, sparq.FORMAT_MXINT8, v)
    return c, s, v.double()


def inputs(seed, M, N, K, pitch=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((M, K), generator=g, device="cuda") * torch.exp(torch.randn((M, 1), generator=g, device="cuda"))
    room = torch.full((M, pitch or ref.up(N, 8)), float("nan"), dtype=torch.bfloat16, device="cuda")
    dy = room[:, :N]
    dy.copy_(torch.randn((M, N), generator=g, device="cuda"))
    return (dy, *kept(x))


def check(dy, v, dw, M, base=None):
    want, size = dy.double().T @ v, dy.double().abs().T @ v.abs()
    tol = (56 + M / 512) * 2.0 ** -23 * size
    if base is not None:
        want = want + base.double()
        tol = tol + 2.0 ** -23 * base.double().abs()
    far = (dw.double() - want).abs() - tol
    assert bool((far <= 0).all()), (float(far.max()), int(far.argmax()))


@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 8, 32), (2, 129, 33), (63, 128, 128), (64, 64, 64), (65, 200, 130), (100, 128, 256), (333, 200, 1000), (511, 256, 512), (513, 7, 515),
                                   (1000, 512, 260), (1024, 300, 2050), (5000, 24, 96), (20000, 128, 1152), (4096, 1024, 1024), (700, 2048, 2304)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_sizes(M, N, K, accumulate):
    dy, c, s, v = inputs(M + N + K, M, N, K)
    dw = torch.randn((N, K), device="cuda") if accumulate else torch.full((N, K), float("nan"), device="cuda")
    base = dw.clone()
    sparq.sparq_wgrad_mx8(dy, c, s, dw, accumulate=accumulate)
    sparq.sparq_check()
    check(dy, v, dw, M, base if accumulate else None)


@pytest.mark.parametrize("N,K", [(24, 40), (130, 250), (520, 300)])
def test_every_number_of_steps(N, K):
    """However the 64-token steps divide among parts and the CTAs of a cluster: the first tokens of one input, 1 to 130 steps, the last
    step short."""
    dy, c, s, v = inputs(N + K, 130 * 64, N, K)
    for steps in range(1, 131):
        M = steps * 64 - steps % 3
        dw = torch.full((N, K), float("nan"), device="cuda")
        sparq.sparq_wgrad_mx8(dy[:M], c[:M], s[:M], dw)
        sparq.sparq_check()
        check(dy[:M], v[:M], dw, M, None)


@pytest.mark.parametrize("M,N,K", [(65536, 256, 256), (100000, 2048, 512)])
def test_long_sums_keep_32_bits(M, N, K):
    """All terms of one sign, where a sum that is cut off instead of rounded drifts: the relative error stays below 2^-19, twice what 48 cut
    additions of a part (half a unit each on average), M / 512 rounded ones and 8 more can cost."""
    g = torch.Generator(device="cuda").manual_seed(3)
    dy = torch.rand((M, N), generator=g, device="cuda").bfloat16()
    c, s, v = kept(torch.rand((M, K), generator=g, device="cuda"))
    dw = torch.empty((N, K), device="cuda")
    sparq.sparq_wgrad_mx8(dy, c, s, dw)
    want = dy.double().T @ v
    assert float(((dw.double() - want).abs() / want).max()) <= 2.0 ** -23 * (56 + M / 512) / 2 + 2.0 ** -24
    assert float((dw.double() - want).norm() / want.norm()) <= 2.0 ** -19


@pytest.mark.parametrize("N,K", [(128, 300), (640, 1024)])
def test_one_hot_tokens(N, K):
    """A token whose dy has a single 1 adds its kept row to one row of dw: every element's place, bit for bit, scales of all sizes."""
    M = 96
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((M, K), generator=g, device="cuda") * 2.0 ** torch.randint(-126, 120, (M, 1), generator=g, device="cuda")
    c, s, v = kept(x)
    dy = torch.zeros((M, N), dtype=torch.bfloat16, device="cuda")
    at = (torch.arange(M, device="cuda") * 37) % N
    assert len(set(at.tolist())) == M
    dy[torch.arange(M, device="cuda"), at] = 1.0
    dw = torch.empty((N, K), device="cuda")
    sparq.sparq_wgrad_mx8(dy, c, s, dw)
    want = torch.zeros((N, K), device="cuda")
    want[at] = v.float()
    assert torch.equal(dw, want)


def test_every_code_and_scale():
    """All 255 codes under the smallest, ordinary and the largest scales."""
    codes = torch.arange(-127, 128, dtype=torch.int8, device="cuda")
    for e in (0, 1, 5, 6, 7, 8, 60, 127, 200, 253, 254):
        c = torch.zeros((1, 256), dtype=torch.int8, device="cuda")
        c[0, :255] = codes
        s = torch.full((1, 16), e, dtype=torch.uint8, device="cuda")
        dy = torch.ones((1, 8), dtype=torch.bfloat16, device="cuda")
        dw = torch.empty((8, 255), device="cuda")
        sparq.sparq_wgrad_mx8(dy, c, s, dw)
        want = (codes.double() * 2.0 ** (e - 127 - 6)).float()
        assert torch.equal(dw, want.expand(8, 255)), e


def test_nan_blocks():
    dy, c, s, v = inputs(4, 70, 40, 200)
    s[5, 2] = 0xFF
    dw = torch.empty((40, 200), device="cuda")
    sparq.sparq_wgrad_mx8(dy, c, s, dw)
    want = torch.zeros((40, 200), dtype=torch.bool, device="cuda")
    want[:, 64:96] = True
    assert torch.equal(torch.isnan(dw), want)


def test_no_tokens_and_pitches():
    c, s = torch.empty((0, 64), dtype=torch.int8, device="cuda"), torch.empty((0, 16), dtype=torch.uint8, device="cuda")
    dw = torch.ones((8, 64), device="cuda")
    dy = torch.empty((0, 8), dtype=torch.bfloat16, device="cuda")
    sparq.sparq_wgrad_mx8(dy, c, s, dw, accumulate=True)
    assert bool((dw == 1).all())
    sparq.sparq_wgrad_mx8(dy, c, s, dw)
    assert not bool(dw.any())
    # dy inside a wider matrix whose other columns are NaN, and outputs at an odd address
    dy, c, s, v = inputs(6, 300, 72, 100, pitch=160)
    room = torch.full((72 * 100 + 8,), 9.0, device="cuda")
    sparq.sparq_wgrad_mx8(dy, c, s, room[1:7201].view(72, 100))
    check(dy, v, room[1:7201].view(72, 100), 300)
    assert room[0] == 9.0 and bool((room[7201:] == 9.0).all())
    with pytest.raises(sparq.SparqError):
        sparq.sparq_wgrad_mx8(torch.zeros((300, 76), dtype=torch.bfloat16, device="cuda")[:, :72], c, s, torch.empty((72, 100), device="cuda"))


@pytest.mark.parametrize("M,N,K", [(9000, 128, 300), (3000, 1024, 1024)])
def test_same_bits_every_time(M, N, K):
    dy, c, s, v = inputs(8, M, N, K)
    got = []
    for _ in range(3):
        got.append(torch.empty((N, K), device="cuda"))
        sparq.sparq_wgrad_mx8(dy, c, s, got[-1])
    assert all(torch.equal(g, got[0]) for g in got)


@pytest.mark.parametrize("M,N,K", [(17356, 2607, 1), (18400, 2675, 3), (20270, 2044, 94), (3499, 4717, 147), (4100, 2560, 2040)])
def test_same_bits_with_cold_caches(M, N, K):
    """Loads that come late and out of order: 300 calls with L2 emptied in between (half of them) give the first call's bits."""
    dy, c, s, v = inputs(9, M, N, K)
    first = torch.empty((N, K), device="cuda")
    sparq.sparq_wgrad_mx8(dy, c, s, first)
    check(dy, v, first, M)
    flush = torch.empty(160 << 18, device="cuda")
    dw, differ = torch.empty((N, K), device="cuda"), torch.zeros((), dtype=torch.int64, device="cuda")
    for i in range(300):
        if i & 1:
            flush.fill_(i)
        sparq.sparq_wgrad_mx8(dy, c, s, dw)
        differ += (dw != first).any()
    sparq.sparq_check()
    assert int(differ) == 0


def test_gradient_against_differences():
    """The loss sum(dy * (X w^T)) is linear in w: its difference quotient over any step is the gradient, up to the rounding of 64 bits."""
    M, N, K = 200, 16, 40
    dy, c, s, v = inputs(2, M, N, K)
    dw = torch.empty((N, K), device="cuda")
    sparq.sparq_wgrad_mx8(dy, c, s, dw)
    w = torch.randn((N, K), device="cuda", dtype=torch.float64)
    loss = lambda w: float((dy.double() * (v @ w.T)).sum())  # noqa: E731
    for n, k in ((0, 0), (7, 39), (15, 20)):
        step = torch.zeros_like(w)
        step[n, k] = 1.0
        size = float((dy[:, n].double() * v[:, k]).abs().sum())
        quotient = (loss(w + step) - loss(w - step)) / 2
        assert abs(quotient - float(dw[n, k])) <= 57 * 2.0 ** -23 * size + 1e-9 * abs(loss(w))
