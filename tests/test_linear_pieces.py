"""What a GPU cannot be asked for about sums in pieces: registers that change hands, and tensor memory of kernels whose CTAs wait for one another while they hold some."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2105_11010_b200", "csrc")


def source(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


def test_registers_of_pairs_add_up_to_what_was_launched():
    """Whole groups of four warps; no more than the launch bound of one block allows."""
    text = source("sparq_linear_kernel.cuh")
    epilogue, others = (int(n) for n in re.findall(r"setmaxnreg\.\w+\.sync\.aligned\.u32 (\d+)", text))
    assert "lin_threads(bool pieces) { return 32 * (pieces ? 4 + kLinEpiWarps : 3 + kLinEpiWarps); }" in text and "constexpr int kLinEpiWarps = 8;" in text
    launched = 65536 // (32 * 12) // 8 * 8
    assert epilogue % 8 == others % 8 == 0 and 8 * epilogue + 4 * others <= 12 * launched


def test_tensor_memory_of_the_clusters_that_share_an_sm():
    """CTAs hold their accumulators while they wait for their cluster: as many as an SM's registers let in, of any launches, must find room, or clusters could wait for one another."""
    text = source("sparq_linear_small_kernel.cuh")
    assert "kCols = tmem_columns(2 * BN);" in text and "lin_small_epi(bool swap) { return swap ? 4 : 8; }" in text and "lin_small_threads(bool swap) { return 32 * (3 + lin_small_epi(swap)); }" in text
    # registers a thread, at the least, that the sums alone take (a lane's columns and the 16 to 64 that are being added)
    share = [max(32, 2 * columns) / (threads * least) for columns, threads, least in ((16, 224, 48), (32, 224, 64), (64, 224, 112), (128, 352, 128))]
    assert 65536 * max(share) <= 512
