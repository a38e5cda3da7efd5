"""sparq_linear's sums over long K: terms of one sign, whose losses add up, and of mixed signs, in every form of launch."""
import pytest
import torch

import paper_2105_11010_b200 as sparq
from ffn_reference import F64, inside, matrix, runs
from test_gpu_linear import experts_rows, room

pytestmark = pytest.mark.gpu

# A sum is cut off, by a unit of 2^-23 of itself at the most, at each addition of 16 products, within pieces of at most so many elements (beside fp32 outputs and kept z 12 sqrt(K), if that is less); the
# pieces are added rounded to nearest.
PIECE = {torch.float32: 1024, torch.float16: 8192, torch.bfloat16: 8192}


def sum_error(size, k, out_type):
    """What a sum of terms whose magnitudes add up to `size` may be off by: its pieces, in up to eight runs of them; the bias."""
    piece = min(k, PIECE[out_type])
    return size * ((piece / 16 + 2) * 2.0 ** -23 + (-(-k // piece) + 8 + 1) * 2.0 ** -24)


def products(x, w, pieces):
    return torch.cat([x[a:b].to(F64) @ w[i].to(F64).T for i, (a, b) in enumerate(pieces)])


# (columns of a tile, CTAs that share one) of sizes (M, N, K, experts)
FORMS = [((16, 1), (8, 4104, 20000, 9)), ((16, 8), (3, 72, 66000, 1)), ((32, 1), (300, 2056, 20000, 9)), ((32, 2), (40, 4104, 20000, 3)), ((64, 1), (520, 2056, 20000, 9)),
         ((64, 4), (130, 2056, 40000, 1)), ((128, 1), (130, 4104, 20008, 3)), ((128, 4), (1, 4104, 40000, 1)), ((256, 1), (520, 4104, 20000, 1)), ((256, 1), (1500, 2056, 9000, 3))]


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("form,size", FORMS)
def test_long_sums(form, size, transposed):
    m, n, k, e = size
    if torch.cuda.get_device_properties(0).multi_processor_count == 148:
        f = sparq.sparq_selftest_linear_form(*size)
        assert (f["columns"], f["split"]) == form
    dt = torch.float16 if m % 20 == 0 else torch.bfloat16
    offsets = experts_rows(m, e, 7) if e > 1 else None
    pieces = runs(offsets) if e > 1 else [(0, m)]
    for one_sign in (True, False):
        g = torch.Generator(device="cuda").manual_seed(m)
        x = torch.randn((m, k), generator=g, device="cuda").to(dt)
        w = torch.randn((e, n, k), generator=g, device="cuda").mul_(k ** -0.5).to(dt)
        if one_sign:
            x, w = x.abs(), w.abs()
        z, size_of = products(x, w, pieces), products(x.abs(), w.abs(), pieces)
        given = w.transpose(1, 2).contiguous() if transposed else w
        call = lambda out, **more: sparq.sparq_linear(x, given if e > 1 else given[0], out, transposed=transposed, offsets=offsets, **more)
        for ot in (torch.float32, dt):
            out = room(m, n, ot)
            call(out)
            inside(out, z, sum_error(size_of, k, ot) + torch.finfo(ot).eps / 2 * z.abs() + 2.0 ** -25)
        del w, given
    sparq.sparq_check()


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("m,n", [(700, 2056), (140, 136), (20, 40)])
def test_what_sums_lose_beside_16_bits(m, n, transposed):
    """Sums of one sign, less a bias of nearly their size, so that the output's rounding hides nothing."""
    k, dt = 200000, torch.bfloat16
    x, w = (torch.rand((rows, k), generator=torch.Generator(device="cuda").manual_seed(rows), device="cuda").add_(0.5).to(dt) for rows in (m, n))
    z = x.to(F64) @ w.to(F64).T
    bias = -z.mean(0).float()
    want = z + bias.to(F64)
    out = room(m, n, dt)
    codes = torch.empty((m, -(-n // 32) * 32), dtype=torch.int8, device="cuda")
    scales = torch.empty((sparq.sparq_mx_scale_bytes(sparq.FORMAT_MXINT8, m, n),), dtype=torch.uint8, device="cuda").view(m, -1)
    sparq.sparq_linear(x, w.T.contiguous() if transposed else w, out, transposed=transposed, bias=bias, z_codes=codes, z_scales=scales)
    off = sum_error(z, k, dt)
    inside(out, want, off + torch.finfo(dt).eps / 2 * (want.abs() + off))
    unit = torch.exp2(scales[:, :codes.shape[1] // 32].to(F64) - 133).repeat_interleave(32, 1)[:, :n]
    inside(codes[:, :n].to(F64) * unit, want, off + torch.where(want.abs() > 127 * unit, unit, unit / 2) * (1 + 2.0 ** -20))
    sparq.sparq_check()


@pytest.mark.parametrize("k", [120, 128, 136, 384, 392, 768, 1023, 1024, 1032, 4104])
@pytest.mark.parametrize("m,n", [(1, 72), (30, 264), (150, 1000), (900, 2056)])
def test_around_the_ends_of_pieces(m, n, k):
    """fp32 outputs in one, two, three and more pieces, with everything that an epilogue does."""
    dt = torch.bfloat16
    x, w, bias, res = matrix(m, k, dt, 1), matrix(n, k, dt, 2, k ** -0.5), torch.randn(n, device="cuda"), matrix(m, n, torch.float32, 3, pitch=n)
    out = room(m, n, torch.float32)
    sparq.sparq_linear(x, w, out, bias=bias, act=1, residual=res)
    size_of = x.to(F64).abs() @ w.to(F64).abs().T + bias.to(F64).abs()
    y = (x.to(F64) @ w.to(F64).T + bias.to(F64)).clamp(min=0.0) + res.to(F64)
    inside(out, y, sum_error(size_of, k, torch.float32) + 2.0 ** -24 * y.abs() + 1e-30)



@pytest.mark.parametrize("m,n,k", [(20, 264, 9000), (150, 1000, 1500), (900, 2056, 1500)])
def test_same_bits_captured_and_on_two_streams(m, n, k):
    dt = torch.bfloat16
    x, w, bias, res = matrix(m, k, dt, 1), matrix(n, k, dt, 2, k ** -0.5), torch.randn(n, device="cuda"), matrix(m, n, torch.float32, 3, pitch=n)

    def step():
        out, half = room(m, n, torch.float32), room(m, n, dt)
        codes = torch.empty((m, -(-n // 32) * 32), dtype=torch.int8, device="cuda")
        scales = torch.empty((sparq.sparq_mx_scale_bytes(sparq.FORMAT_MXINT8, m, n),), dtype=torch.uint8, device="cuda")
        sparq.sparq_linear(x, w, out, bias=bias, act=3, residual=res)
        sparq.sparq_linear(x, w, half, bias=bias, act=2, z_codes=codes, z_scales=scales)
        return out, half, codes, scales

    first = step()
    streams, others = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(4):
        for s in streams:
            with torch.cuda.stream(s):
                others.append(step())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        recorded = step()
    for t in recorded:
        t.zero_()
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    for other in others + [recorded]:
        assert all(torch.equal(a, b) for a, b in zip(first, other))
    sparq.sparq_check()
