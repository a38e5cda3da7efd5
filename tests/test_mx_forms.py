"""Which form the microscaled contractions take (host-side rules on the sizes), without a device."""
import pytest

import paper_2105_11010_b200 as sparq

SCRATCH = 1 << 30          # the most scratch memory that a call gets
TOKENS = [1, 63, 64, 65, 333, 511, 1000, 4096, 10000, 16384, 32768, 65536, 100352, 131072, 200000, 1 << 20, 1 << 24, (1 << 31) - 257]
SIZES = [1, 8, 100, 128, 257, 512, 1152, 2048, 2560, 4096, 5120, 8192, 16384, 65536, 1 << 20, (1 << 31) - 257]


@pytest.mark.parametrize("M", TOKENS)
def test_a_weight_gradient_gets_the_scratch_of_its_form(M):
    """A form is chosen by what it costs with its scratch memory, so that has to be had: X in bf16 and the parts' sums are one piece."""
    for N in SIZES:
        for K in SIZES:
            f = sparq.sparq_selftest_wgrad_form(M, N, K)
            assert 0 <= f["scratch_bytes"] <= SCRATCH, (M, N, K, f)


@pytest.mark.parametrize("M,N,K", [(131072, 4096, 4096), (131072, 2048, 4096), (65536, 8192, 8192), (32768, 5120, 16384), (100000, 4096, 5000)])
def test_sums_beside_a_large_x(M, N, K):
    """X in bf16 takes the whole of it, or all but what a last round's sums would need: neither is lost with the other."""
    f = sparq.sparq_selftest_wgrad_form(M, N, K)
    assert f["kernel"] in (1, 2) and f["scratch_bytes"] <= SCRATCH
    if M * K * 2 == SCRATCH:
        assert f["kernel"] == 2 and f["whole"] == 0 and f["scratch_bytes"] == SCRATCH


@pytest.mark.parametrize("M", [1, 64, 333, 5000, 100352])
def test_parts_and_clusters_have_steps_for_everyone(M):
    for N in SIZES[:-2]:
        for K in SIZES[:-2]:
            f, blocks = sparq.sparq_selftest_wgrad_form(M, N, K), -(-M // 64)
            assert 1 <= f["parts"] * f["split"] <= blocks and 0 <= f["whole"] < f["tiles"], (M, N, K, f)
            tile = 256 if f["kernel"] else 128
            assert f["tiles"] == -(-N // tile) * -(-K // tile)


def test_bad_sizes_are_refused():
    for args in ((0, 1, 1), (1, -1, 1), (1, 1, 1 << 31), (1, 1, 1, 0)):
        with pytest.raises(sparq.SparqError) as e:
            sparq.sparq_selftest_wgrad_form(*args)
        assert e.value.code == -1


@pytest.mark.parametrize("sms", range(1, 161))
def test_devices_of_few_multiprocessors(sms):
    """A process may be given a share of a device: clusters that do not fit are not chosen, nor divided by."""
    fits = {1: sms, 2: sms // 2, 4: sms // 4, 8: sms // 8}
    for M in (1, 20, 100, 1000):
        for N in (64, 4096):
            for K in (64, 2048, 16384):
                f = sparq.sparq_selftest_mxf4_form(M, N, K, sms)
                assert fits[2 if f["columns"] == 256 else f["split"]] > 0, (M, N, K, f)
                f = sparq.sparq_selftest_wgrad_form(K, N, M, sms)
                assert fits[2 if f["kernel"] else f["split"]] > 0, (M, N, K, f)


def test_forms_of_products():
    """Rows of A in columns up to 32 of them, and pairs for large grids."""
    assert sparq.sparq_selftest_mxf4_form(1, 4096, 4096)["columns"] == 16
    assert sparq.sparq_selftest_mxf4_form(17, 4096, 4096)["columns"] == 32
    assert sparq.sparq_selftest_mxf4_form(16384, 4096, 4096) == {"columns": 256, "split": 1, "tiles": 64 * 16}
    for args in ((0, 1, 1), (1, 1 << 31, 1), (1, 1, 1, 0)):
        with pytest.raises(sparq.SparqError) as e:
            sparq.sparq_selftest_mxf4_form(*args)
        assert e.value.code == -1
