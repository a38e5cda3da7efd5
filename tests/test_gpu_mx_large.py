"""The persistent forms of the microscaled contractions, with several tiles to a pair of CTAs and ragged edges.  Operands are
quantized by the library (tested by itself), references are 64-bit products on the device; tolerances as in test_gpu_mx_gemm.py and
test_gpu_mx_wgrad.py."""
import pytest
import torch

import mx_reference as ref
import paper_2105_11010_b200 as sparq

pytestmark = pytest.mark.gpu

# NVFP4's tensor scale is 1 for this largest magnitude, so that decoded values are exact in fp32
UNIT = 2688.0


def operand(x, fmt):
    rows, cols = x.shape
    c = torch.empty((rows, ref.up(cols, 32) // 2), dtype=torch.uint8, device="cuda")
    s = torch.empty(sparq.sparq_mx_scale_bytes(fmt, rows, cols), dtype=torch.uint8, device="cuda")
    m = torch.tensor([UNIT], device="cuda") if fmt == ref.NVFP4 else None
    sparq.sparq_quantize_mx(x, fmt, c, s, max_dev=m)
    v = torch.empty((rows, cols), device="cuda")
    sparq.sparq_dequantize_mx(c, s, fmt, v, max_dev=m)
    return c, s, v.double(), m


def product(a, b, fmt, **kw):
    if fmt == ref.NVFP4:
        kw.update(a_max=a[3], b_max=b[3])
    sparq.sparq_gemm_mxf4(a[0], a[1], b[0], b[1], fmt, **kw)


@pytest.mark.parametrize("fmt", [ref.MXFP4, ref.NVFP4])
@pytest.mark.parametrize("M,N,K", [(4000, 2304, 384), (4001, 2305, 96), (2050, 5000, 1000), (300, 20000, 4160)])
@pytest.mark.parametrize("bias", [False, True])
def test_products(fmt, M, N, K, bias):
    g = torch.Generator(device="cuda").manual_seed(M + N)
    a = operand(torch.randn((M, K), generator=g, device="cuda") * 100, fmt)
    b = operand(torch.randn((N, K), generator=g, device="cuda") * 100, fmt)
    bi = torch.randn(N, generator=g, device="cuda") * 1e4 if bias else None
    f = torch.full((M, N), float("nan"), device="cuda")
    h = torch.full((M, N), float("nan"), dtype=torch.bfloat16, device="cuda")
    product(a, b, fmt, bias=bi, f32_out=f)
    product(a, b, fmt, bias=bi, bf16_out=h, relu=True)
    sparq.sparq_check()
    y = a[2] @ b[2].T
    tol = (K / 64 + 72) * 2.0 ** -23 * (a[2].abs() @ b[2].abs().T)
    if bias:
        y = y + bi.double()
    tol = tol + 4 * 2.0 ** -24 * (y.abs() + (bi.double().abs() if bias else 0.0))
    assert bool(((f.double() - y).abs() <= tol).all())
    y = y.clamp(min=0.0)
    assert bool(((h.double() - y).abs() <= tol + 2.0 ** -8 * (y + tol)).all())


@pytest.mark.parametrize("fmt", [ref.MXFP4, ref.NVFP4])
def test_one_hot_rows_and_nan_blocks(fmt):
    """Every element's place, and NaN in its own rows and columns only."""
    M, N, K = 4000, 2304, 544
    b = operand(torch.randn((N, K), device="cuda") * 100, fmt)
    at = (torch.arange(M, device="cuda") * 7) % K
    x = torch.zeros((M, K), device="cuda")
    x[torch.arange(M, device="cuda"), at] = 1.0
    a = operand(x, fmt)
    f = torch.empty((M, N), device="cuda")
    product(a, b, fmt, f32_out=f)
    want = b[2].T[at].float() * a[2][torch.arange(M, device="cuda"), at].float()[:, None]
    assert torch.equal(f, want)
    x[M - 1, K - 1] = float("nan")
    x[257, 0] = float("inf")
    w = torch.randn((N, K), device="cuda")
    w[300, 100] = float("nan")
    product(operand(x, fmt), operand(w, fmt), fmt, f32_out=f)
    nan = torch.zeros((M, N), dtype=torch.bool, device="cuda")
    nan[M - 1] = nan[257] = nan[:, 300] = True
    assert torch.equal(torch.isnan(f), nan)


@pytest.mark.parametrize("N", [2304, 2305])
def test_nothing_behind_the_last_row(N):
    M, K = 4001, 64
    a, b = operand(torch.randn((M, K), device="cuda"), 0), operand(torch.randn((N, K), device="cuda"), 0)
    f = torch.full((M * N + 4096,), 5.0, device="cuda")
    h = torch.full((M * N + 4096,), 5.0, dtype=torch.bfloat16, device="cuda")
    product(a, b, 0, f32_out=f[:M * N].view(M, N), bf16_out=h[:M * N].view(M, N))
    assert bool((f[M * N:] == 5.0).all()) and bool((h[M * N:] == 5.0).all())


def kept(x):
    rows, cols = x.shape
    c = torch.empty((rows, ref.up(cols, 32)), dtype=torch.int8, device="cuda")
    s = torch.empty((rows, ref.up(ref.up(cols, 32) // 32, 16)), dtype=torch.uint8, device="cuda")
    sparq.sparq_quantize_mx(x, sparq.FORMAT_MXINT8, c, s)
    v = torch.empty((rows, cols), device="cuda")
    sparq.sparq_dequantize_mx(c, s, sparq.FORMAT_MXINT8, v)
    return c, s, v.double()


# one part and several, both tile sizes, expanded first and not, tiles of a last round in parts (the last four)
WGRADS = [(200, 2304, 2304), (6000, 2600, 2600), (5000, 1000, 1100), (30000, 300, 700), (9001, 72, 300), (40000, 128, 1152), (3000, 4100 // 8 * 8, 513),
          (4100, 2560, 2040), (2500, 2504, 2003), (1500, 2490, 2001), (4096, 4096, 4096)]


@pytest.mark.parametrize("M,N,K", WGRADS)
@pytest.mark.parametrize("accumulate", [False, True])
def test_weight_gradients_captured_and_with_a_workspace(M, N, K, accumulate):
    """The same bits eagerly, with a workspace, captured without one and captured with one."""
    g = torch.Generator(device="cuda").manual_seed(M + N + K)
    c, s, v = kept(torch.randn((M, K), generator=g, device="cuda"))
    dy = torch.zeros((M, ref.up(N, 8)), dtype=torch.bfloat16, device="cuda")[:, :N]      # rows of 16-byte pieces
    dy.copy_(torch.randn((M, N), generator=g, device="cuda"))
    base = torch.randn((N, K), generator=g, device="cuda") if accumulate else torch.full((N, K), float("nan"), device="cuda")
    dw = base.clone()
    sparq.sparq_wgrad_mx8(dy, c, s, dw, accumulate=accumulate)
    sparq.sparq_check()
    want, size = dy.double().T @ v, dy.double().abs().T @ v.abs()
    if accumulate:
        want, size = want + base.double(), size + base.double().abs()
    # 56 and M / 512 additions, and one for each of up to 128 parts
    assert bool(((dw.double() - want).abs() <= (56 + M / 512 + 128) * 2.0 ** -23 * size).all())
    need = sparq.sparq_wgrad_mx8_workspace_bytes(M, N, K)
    ws = torch.full((max(need, 1),), 0xFF, dtype=torch.uint8, device="cuda")
    got = base.clone()
    sparq.sparq_wgrad_mx8(dy, c, s, got, accumulate=accumulate, workspace=ws)
    assert torch.equal(got, dw)
    for w in (None, ws):
        got = base.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            sparq.sparq_wgrad_mx8(dy, c, s, got, accumulate=accumulate, workspace=w)
        got.copy_(base)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, dw)
        if accumulate:
            graph.replay()
            again = dw.clone()
            sparq.sparq_wgrad_mx8(dy, c, s, again, accumulate=True)
            assert torch.equal(got, again)
    if need:
        with pytest.raises(sparq.SparqError):
            sparq.sparq_wgrad_mx8(dy, c, s, got, workspace=ws[:need - 1])


@pytest.mark.parametrize("N,K", [(2304, 2304), (128, 1152), (1000, 1100)])
def test_tokens_land_on_their_rows(N, K):
    """One-hot tokens, in every form: dw is the kept rows, bit for bit."""
    M = min(N, 2000)
    c, s, v = kept(torch.randn((M, K), device="cuda") * 2.0 ** torch.randint(-100, 100, (M, 1), device="cuda"))
    at = torch.randperm(N, device="cuda")[:M]
    dy = torch.zeros((M, N), dtype=torch.bfloat16, device="cuda")
    dy[torch.arange(M, device="cuda"), at] = 1.0
    dw = torch.empty((N, K), device="cuda")
    sparq.sparq_wgrad_mx8(dy, c, s, dw)
    want = torch.zeros((N, K), device="cuda")
    want[at] = v.float()
    assert torch.equal(dw, want)
