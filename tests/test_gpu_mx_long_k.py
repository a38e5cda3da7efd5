"""4-bit products over a long reduction whose terms have one sign, where sums that are cut off drift.

The tensor cores add 64 products to a running sum in fp32 and cut the sum off below its 24 bits.  Of K / 64 additions of terms of one sign
and about one size the i-th leaves less than 2^-23 of i / (K / 64) of the result: K / 128 units of 2^-23 in all, and 72 for the additions within a step,
the partial sums of a split and the epilogue, as in test_gpu_mx_gemm.py."""
import pytest
import torch

import mx_reference as ref
import paper_2105_11010_b200 as sparq

pytestmark = pytest.mark.gpu

UNIT = 2688.0          # NVFP4's tensor scale is 1 for this largest magnitude


def operand(rows, cols, fmt, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.rand((rows, cols), generator=g, device="cuda") + 0.5
    x *= 2.0 ** -torch.randint(0, 8, (rows, ref.up(cols, 32) // 32), generator=g, device="cuda").float().repeat_interleave(32, 1)[:, :cols]
    c = torch.empty((rows, ref.up(cols, 32) // 2), dtype=torch.uint8, device="cuda")
    s = torch.empty(sparq.sparq_mx_scale_bytes(fmt, rows, cols), dtype=torch.uint8, device="cuda")
    m = torch.tensor([UNIT], device="cuda") if fmt == ref.NVFP4 else None
    if fmt == ref.NVFP4:
        x = x * UNIT / 2
    sparq.sparq_quantize_mx(x, fmt, c, s, max_dev=m)
    v = torch.empty((rows, cols), device="cuda")
    sparq.sparq_dequantize_mx(c, s, fmt, v, max_dev=m)
    return c, s, v.double(), m


@pytest.mark.parametrize("fmt", [ref.MXFP4, ref.NVFP4])
@pytest.mark.parametrize("M,N,K,columns,split", [(1, 30000, 65536, 16, 1), (1, 128, 65536, 16, 8), (30, 700, 40000, 32, 8), (200, 300, 65536, 128, 8),
                                                 (2304, 2304, 32768, 256, 1), (400, 4096, 65536, 256, 1)])
def test_one_sign(fmt, M, N, K, columns, split):
    form = sparq.sparq_selftest_mxf4_form(M, N, K, torch.cuda.get_device_properties(0).multi_processor_count)
    assert (form["columns"], form["split"]) == (columns, split)
    a, b = operand(M, K, fmt, 1), operand(N, K, fmt, 2)
    out = torch.empty((M, N), device="cuda")
    kw = dict(a_max=a[3], b_max=b[3]) if fmt == ref.NVFP4 else {}
    sparq.sparq_gemm_mxf4(a[0], a[1], b[0], b[1], fmt, f32_out=out, **kw)
    sparq.sparq_check()
    want = a[2] @ b[2].T
    norm = float((out.double() - want).norm() / want.norm())
    print(f"{M} x {N} x {K}: 2-norm {norm:.2e}, sign {float(((out.double() - want) / want).mean()):.2e}")
    assert bool(((out.double() - want).abs() <= (K / split / 128 + 72) * 2.0 ** -23 * want).all())
    assert norm <= (K / split / 128 + 72) * 2.0 ** -23
