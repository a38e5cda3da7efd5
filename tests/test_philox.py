"""The tests' restatement of Philox4x32-10 against the answers that its authors publish with it (Random123's known-answer vectors), and the order in which dropout takes its bits."""
import numpy as np
import pytest

from ffn_reference import kept, philox

# counter, key, answer
KNOWN = [((0x00000000,) * 4, (0x00000000,) * 2, (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
         ((0xffffffff,) * 4, (0xffffffff,) * 2, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
         ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0), (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1))]


@pytest.mark.parametrize("counter,key,answer", KNOWN)
def test_known_answers(counter, key, answer):
    assert tuple(int(w) for w in philox(counter, key)) == answer


def test_the_first_block_of_dropout():
    """Seed 0, draw 0, row 0: the first known answer's halves, low half first; an element is kept where its half is at least 65536 p."""
    halves = np.array(KNOWN[0][2], dtype="<u4").view("<u2")
    for p in (0.1, 0.5, 0.875):
        keep, _ = kept(1, 8, p, 0, 0)
        assert keep[0].tolist() == [int(h) >= int(65536 * p + 0.5) for h in halves]


@pytest.mark.gpu
def test_the_kernel_draws_the_known_block():
    import torch

    import paper_2105_11010_b200 as sparq

    halves = np.array(KNOWN[0][2], dtype="<u4").view("<u2")
    x, out = torch.ones((1, 8), device="cuda"), torch.empty((1, 8), device="cuda")
    for p in (0.1, 0.5, 0.875):
        sparq.sparq_dropout(x, p, torch.zeros(2, dtype=torch.int64, device="cuda"), out)
        assert (out[0] != 0).tolist() == [int(h) >= int(65536 * p + 0.5) for h in halves]
