"""A row's outputs of sparq_linear depend on that row alone: not on the rows beside it, nor on what lies behind an expert's rows, to the last bit."""
import pytest
import torch

import paper_2105_11010_b200 as sparq
from ffn_reference import matrix
from test_gpu_linear import room, runs

pytestmark = pytest.mark.gpu

# (columns of a tile, CTAs that share one) of sizes (M, N, K, experts); fp16, whose rounding lets most of a sum's and an activation's last bits through
FORMS = [((16, 1), (8, 4104, 72, 9)), ((16, 8), (7, 2056, 1000, 1)), ((32, 1), (40, 4104, 72, 3)), ((32, 2), (40, 4104, 2048, 3)), ((64, 1), (2100, 520, 72, 40)),
         ((64, 4), (130, 2056, 2048, 1)), ((128, 1), (520, 72, 72, 3)), ((128, 2), (130, 2056, 1000, 3)), ((256, 1), (2300, 4104, 72, 1)), ((256, 1), (2300, 1000, 136, 7))]
SEEDS = 6


def of_form(form, size):
    if torch.cuda.get_device_properties(0).multi_processor_count == 148:
        f = sparq.sparq_selftest_linear_form(*size)
        assert (f["columns"], f["split"]) == form


def weights(n, k, e, seed):
    return matrix(e * n, k, torch.float16, seed, k ** -0.5).unflatten(0, (e, n))


def strange(x, rows, seed):
    """Rows whose products are not numbers, or far below what an activation function leaves of them."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x[rows] = torch.randn(x[rows].shape, generator=g, device="cuda").mul_(300.0).to(x.dtype)
    x[rows[::3]] = float("nan")


@pytest.mark.parametrize("act", [2, 3])
@pytest.mark.parametrize("form,size", FORMS)
def test_in_any_order(form, size, act):
    m, n, k, e = size
    of_form(form, size)
    for seed in range(SEEDS):
        x, w, bias = matrix(m, k, torch.float16, seed), weights(n, k, e, seed + 100), torch.randn((e, n), device="cuda")
        strange(x, torch.arange(3, m, 5, device="cuda"), seed)
        offsets = (torch.arange(e + 1, device="cuda") * m // e).to(torch.int32) if e > 1 else None
        order = torch.cat([a + torch.randperm(b - a) for a, b in (runs(offsets) if e > 1 else [(0, m)])]).cuda()
        here, there = room(m, n, torch.float16), room(m, n, torch.float16)
        call = lambda x, out: sparq.sparq_linear(x, w if e > 1 else w[0], out, bias=bias if e > 1 else bias[0], act=act, offsets=offsets)
        call(x, here)
        call(x[order], there)
        there, here = there.view(torch.int16), here[order].view(torch.int16)
        plain = ~torch.isnan(x[order, 0])       # (a NaN's bits are free)
        assert torch.equal(there[plain], here[plain])


@pytest.mark.parametrize("act", [2, 3])
@pytest.mark.parametrize("form,size", [f for f in FORMS if f[1][3] > 1])
def test_whatever_lies_behind_the_last_run(form, size, act):
    m, n, k, e = size
    of_form(form, size)
    first, last = m // 9, m - m // 5
    offsets = (first + torch.arange(e + 1, device="cuda") * (last - first) // e).to(torch.int32)
    others = torch.cat([torch.arange(first), torch.arange(last, m)]).cuda()
    for seed in range(SEEDS):
        x, w = matrix(m, k, torch.float16, seed), weights(n, k, e, seed + 100)
        x[others] = 0.0
        clean, out = room(m, n, torch.float16), room(m, n, torch.float16)
        sparq.sparq_linear(x, w, clean, act=act, offsets=offsets)
        strange(x, others, seed)
        sparq.sparq_linear(x, w, out, act=act, offsets=offsets)
        assert torch.equal(out, clean)
