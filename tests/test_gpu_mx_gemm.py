"""Products of 4-bit microscaled operands against 64-bit products of what the codes stand for.

Tolerance.  Products of two 4-bit values and two scales are exact.  The tensor cores add the 64 products of a step at a common exponent
and the step to the running sum; each of the K / 64 + 64 additions that an output sees is off by less than a unit of the
last of 24 bits of the largest partial sum, which sum |a b| bounds: (K / 64 + 64 + 8) 2^-23 sum |a b|, the 8 for the partial
sums of a split reduction.  Behind it up to four roundings in fp32 (two quotients' product, the scaling, the bias): 4 * 2^-24 of the
result and of the bias, and half a step of bf16, 2^-8 of the result."""
import numpy as np
import pytest
import torch

import mx_reference as ref
import paper_2105_11010_b200 as sparq

pytestmark = pytest.mark.gpu


def operand(seed, rows, cols, fmt):
    rng = np.random.default_rng(seed)
    x = (rng.standard_normal((rows, cols)) * np.exp(rng.standard_normal((1, cols)))).astype(np.float32)
    m = float(np.abs(x).max()) if x.size else 1.0
    codes, scales, v = ref.device(x, fmt, m)
    return codes, scales, v, m


def run(M, N, K, fmt, bias=False, relu=False, outs=("f32",), seed=0):
    a, sa, va, am = operand(seed + 1, M, K, fmt)
    b, sb, vb, bm = operand(seed + 2, N, K, fmt)
    bi = torch.from_numpy(np.random.default_rng(seed + 3).standard_normal(N).astype(np.float32) * K ** 0.5).cuda() if bias else None
    nv = fmt == ref.NVFP4
    args = dict(bias=bi, relu=relu)
    if nv:
        args.update(a_max=torch.tensor([am], device="cuda"), b_max=torch.tensor([bm], device="cuda"))
    got = {}
    if "f32" in outs:
        got["f32_out"] = torch.full((M, N), 77.0, device="cuda")
    if "bf16" in outs:
        got["bf16_out"] = torch.full((M, N), 77.0, dtype=torch.bfloat16, device="cuda")
    sparq.sparq_gemm_mxf4(a, sa, b, sb, fmt, **args, **got)
    sparq.sparq_check()
    alpha = float(ref.tensor_scale(am)) * float(ref.tensor_scale(bm)) if nv else 1.0
    y = va @ vb.T * alpha
    tol = (K / 64 + 72) * 2.0 ** -23 * (np.abs(va) @ np.abs(vb).T) * alpha + 4 * 2.0 ** -24 * np.abs(y)
    if bias:
        y = y + bi.cpu().numpy().astype(np.float64)
        tol = tol + 4 * 2.0 ** -24 * (np.abs(y) + np.abs(bi.cpu().numpy()))
    y = np.maximum(y, 0) if relu else y
    for name, t in got.items():
        more = 2.0 ** -8 * (np.abs(y) + tol) if name == "bf16_out" else 0.0
        far = np.abs(t.float().cpu().numpy().astype(np.float64) - y) - tol - more
        assert far.max() <= 0, (name, far.max(), np.unravel_index(far.argmax(), far.shape))
    return got


@pytest.mark.parametrize("fmt", [ref.MXFP4, ref.NVFP4])
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 128, 64), (1, 129, 100), (2, 257, 256), (15, 128, 257), (16, 300, 2048), (17, 64, 96), (32, 130, 513), (33, 200, 320), (64, 128, 128),
                                   (65, 77, 640), (128, 128, 1024), (129, 129, 1000), (250, 501, 1000), (256, 256, 4096), (300, 100, 32), (513, 260, 800)])
def test_sizes(fmt, M, N, K):
    run(M, N, K, fmt)


@pytest.mark.parametrize("fmt", [ref.MXFP4, ref.NVFP4])
@pytest.mark.parametrize("M,N,K", [(1, 515, 2050), (40, 96, 256), (257, 384, 700), (600, 1024, 512)])
@pytest.mark.parametrize("bias,relu", [(True, False), (False, True), (True, True)])
def test_epilogue(fmt, M, N, K, bias, relu):
    run(M, N, K, fmt, bias, relu, ("f32", "bf16"))
    run(M, N, K, fmt, bias, relu, ("bf16",))


@pytest.mark.parametrize("fmt", [ref.MXFP4, ref.NVFP4])
def test_large_grid_with_ragged_edges(fmt):
    """Several rounds of tiles: 1029 x 9 column tiles and rows that end inside a tile."""
    run(2100, 2050, 384, fmt, outs=("f32", "bf16"))


@pytest.mark.parametrize("fmt", [ref.MXFP4, ref.NVFP4])
@pytest.mark.parametrize("M", [1, 64, 300])
def test_one_hot_rows_pick_columns(fmt, M):
    """A row with a single 1 (exact in both formats) returns the other operand's column: every element's place in the tiles, bit for bit."""
    K, N = 1024, 300
    b, sb, vb, bm = operand(11, N, K, fmt)
    for shift in (0, 437):
        at = (np.arange(M) * 7 + shift) % K
        x = np.zeros((M, K), np.float32)
        x[np.arange(M), at] = 1.0
        a, sa, va = ref.device(x, fmt, 1.0)
        out = torch.empty((M, N), device="cuda")
        mx = dict(a_max=torch.tensor([1.0], device="cuda"), b_max=torch.tensor([bm], device="cuda")) if fmt == ref.NVFP4 else {}
        sparq.sparq_gemm_mxf4(a, sa, b, sb, fmt, f32_out=out, **mx)
        want = (va @ vb.T).astype(np.float32)               # one product each: exact
        if fmt == ref.NVFP4:
            want = want * (ref.tensor_scale(1.0) * ref.tensor_scale(bm))
        assert np.array_equal(out.cpu().numpy(), want)


@pytest.mark.parametrize("fmt", [ref.MXFP4, ref.NVFP4])
@pytest.mark.parametrize("M,N,K", [(1, 200, 1000), (300, 200, 1000)])
def test_scales_of_each_block(fmt, M, N, K):
    """Scales that differ by powers of two from block to block and row to row, over a wide range."""
    rng = np.random.default_rng(5)
    x = rng.standard_normal((M, K)) * 2.0 ** rng.integers(-6, 7, (M, ref.up(K, 32) // 32)).repeat(32, 1)[:, :K]
    w = rng.standard_normal((N, K)) * 2.0 ** rng.integers(-6, 7, (N, ref.up(K, 32) // 32)).repeat(32, 1)[:, :K]
    am, bm = float(np.abs(x).max()), float(np.abs(w).max())
    a, sa, va = ref.device(x.astype(np.float32), fmt, am)
    b, sb, vb = ref.device(w.astype(np.float32), fmt, bm)
    out = torch.empty((M, N), device="cuda")
    mx = dict(a_max=torch.tensor([am], device="cuda"), b_max=torch.tensor([bm], device="cuda")) if fmt == ref.NVFP4 else {}
    sparq.sparq_gemm_mxf4(a, sa, b, sb, fmt, f32_out=out, **mx)
    alpha = float(ref.tensor_scale(am)) * float(ref.tensor_scale(bm)) if fmt == ref.NVFP4 else 1.0
    y, tol = va @ vb.T * alpha, (K / 64 + 72) * 2.0 ** -23 * (np.abs(va) @ np.abs(vb).T) * alpha
    assert (np.abs(out.cpu().numpy() - y) <= tol + 4 * 2.0 ** -24 * np.abs(y)).all()


@pytest.mark.parametrize("fmt", [ref.MXFP4, ref.NVFP4])
@pytest.mark.parametrize("M", [3, 200, 700])
def test_nan_blocks_reach_their_rows_and_columns_only(fmt, M):
    N, K = 300, 400
    rng = np.random.default_rng(8)
    x, w = rng.standard_normal((M, K)).astype(np.float32), rng.standard_normal((N, K)).astype(np.float32)
    x[M - 1, 399], w[129, 0] = np.nan, np.inf
    a, sa, va = ref.device(x, fmt, 5.0)
    b, sb, vb = ref.device(w, fmt, 5.0)
    out = torch.empty((M, N), device="cuda")
    mx = {k: torch.tensor([5.0], device="cuda") for k in ("a_max", "b_max")} if fmt == ref.NVFP4 else {}
    sparq.sparq_gemm_mxf4(a, sa, b, sb, fmt, f32_out=out, **mx)
    nan = torch.isnan(out).cpu().numpy()
    want = np.zeros((M, N), bool)
    want[M - 1, :] = want[:, 129] = True
    assert np.array_equal(nan, want)


@pytest.mark.parametrize("M,N,K", [(1, 300, 4096), (130, 200, 2048), (1000, 512, 320)])
def test_same_bits_every_time(M, N, K):
    got = [run(M, N, K, ref.NVFP4)["f32_out"] for _ in range(3)]
    assert all(torch.equal(g, got[0]) for g in got)


def test_outputs_stay_within_their_rows():
    """Nothing is written behind the last row."""
    for M, N, K in ((3, 70, 64), (300, 70, 64), (1030, 264, 64)):
        a, sa, va, _ = operand(1, M, K, 0)
        b, sb, vb, _ = operand(2, N, K, 0)
        room = torch.full((M * N + 4096,), 5.0, device="cuda")
        half = torch.full((M * N + 4096,), 5.0, dtype=torch.bfloat16, device="cuda")
        sparq.sparq_gemm_mxf4(a, sa, b, sb, 0, f32_out=room[:M * N].view(M, N), bf16_out=half[:M * N].view(M, N))
        assert bool((room[M * N:] == 5.0).all()) and bool((half[M * N:] == 5.0).all())
        tol = (K / 64 + 72) * 2.0 ** -23 * (np.abs(va) @ np.abs(vb).T)
        assert (np.abs(room[:M * N].view(M, N).cpu().numpy() - va @ vb.T) <= tol).all()


def test_odd_output_addresses():
    """Outputs at any element, whatever the vector stores would like."""
    M, N, K = 260, 96, 128
    a, sa, va, _ = operand(1, M, K, 0)
    b, sb, vb, _ = operand(2, N, K, 0)
    tol = (K / 64 + 72) * 2.0 ** -23 * (np.abs(va) @ np.abs(vb).T)
    for off in (0, 1, 2, 4, 8):
        f = torch.zeros(M * N + 8, device="cuda")[off:off + M * N].view(M, N)
        h = torch.zeros(M * N + 8, dtype=torch.bfloat16, device="cuda")[off:off + M * N].view(M, N)
        sparq.sparq_gemm_mxf4(a, sa, b, sb, 0, f32_out=f, bf16_out=h)
        y = va @ vb.T
        assert (np.abs(f.cpu().numpy() - y) <= tol).all()
        assert (np.abs(h.float().cpu().numpy() - y) <= tol + 2.0 ** -8 * (np.abs(y) + tol)).all()
