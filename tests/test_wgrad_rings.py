"""Rings of the weight gradients' kernels that teams of warps take turns on.

A parity answers for every second phase of a barrier: a team may ask for a phase only when the one before is known to have completed.  A
team knows the phases that it has waited for itself, so a barrier of the X stages, which says that the MMA which read one has retired, has
to be the same team's every time: where teams take turns on a stage there are two sets of them.  (Arrivals on two barriers, the second CTA's remote ones among them, are in no order that anything promises.)
That is a race on shared memory, so it is looked for in the source and in a model of the ring."""
import os
import re

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2105_11010_b200", "csrc")


def source():
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "sparq_wgrad_kernel.cuh")).read())


def rings():
    """(name, raw stages, X stages, teams, sets of X barriers) of both kernels that transform X on the way."""
    src = source()
    pair = re.search(r"struct WgradPair : (\w+(?:<\d+, \d+>)?)", src).group(1)
    pair = re.search(r"using %s = (WgradCta<\d+, \d+>);" % pair, src).group(1) if "<" not in pair else pair
    small = re.search(r"struct WgradSmall : (WgradCta<\d+, \d+>)", src).group(1)
    numbers = lambda t: tuple(int(n) for n in re.findall(r"\d+", t))
    workers = int(re.search(r"kWgPairWorkers = (\d+)", src).group(1))
    sets = int(re.search(r"kWgXSets = (\d+)", src).group(1)) if "kWgXSets" in src else 1
    return [("pair", *numbers(pair), workers // 4, sets), ("small", *numbers(small), int(re.search(r"kWgTeams = (\d+)", src).group(1)), 1)]


def test_a_barrier_of_x_belongs_to_one_team():
    for name, raw, x, teams, sets in rings():
        assert sets * x % teams == 0 and x <= raw, name


def test_the_compiler_is_told():
    src = source()
    assert 'static_assert(X <= R,' in src
    assert 'static_assert(kXBars % kWgPairTeams == 0 && kXBars <= kMaxStages,' in src and "if (stage % kWgPairTeams == team) {" in src
    assert 'static_assert(kX % kWgTeams == 0,' in src and "if (it % kWgTeams == team) {" in src


def test_x_is_waited_for_before_codes():
    """In both workers: the raw stage's wait comes behind the X stage's, which lies behind the raw stage's last use."""
    src = source()
    asked = re.findall(r"mbar_wait_warp\(lane == 0 \? 1u : 0u, (x_empty_bar\([^,]*\), [^,]*|raw_bar\(raw\.s\), raw\.ph),", src)
    assert [a.split("(")[0] for a in asked] == ["x_empty_bar", "raw_bar"] * 2
    assert len(re.findall(r">= kX(?:\)| &&) !?mbar_wait_warp\(lane == 0 \? 1u : 0u, x_empty_bar", src)) == 2


def test_pairs_ask_two_sets_of_x_barriers():
    src = source()
    pair = src[src.index("struct WgradPair :"):]
    assert "kXBars = kWgXSets * kX;" in pair and pair.count("RingAt<kXBars> xe;") == 2 and pair.count("xe.next();") == 2
    assert "tc_commit_pair(x_empty_bar(xe.s), elected);" in pair and "q < Cta::kXBars; ++q) mbar_init(c.x_empty_bar(q), 1);" in pair
    assert "const bool wrap = xe.s < kX;" in pair and "x_empty_bar(wrap ? xe.s + kXBars - kX : xe.s - kX), wrap ? xe.ph ^ 1u : xe.ph," in pair


@pytest.mark.parametrize("x,sets", [(3, 2), (4, 1), (4, 2), (2, 3)])
def test_barrier_and_phase_of_the_step_before(x, sets):
    """What the worker computes from its place in the ring of barriers, for step - x."""
    bars = x * sets
    for step in range(x, 200):
        s, ph = step % bars, step // bars & 1
        wrap = s < x
        at, parity = (s + bars - x, ph ^ 1) if wrap else (s - x, ph)
        assert (at, parity) == ((step - x) % bars, (step - x) // bars & 1)


def model(raw, x, teams, seed, sets=1, trials=2000):
    """How often a team that asks, in the kernels' order, for what its next step needs is told that it is there when it is not.

    MMAs retire in order; their arrivals on the barriers of the X stages, and copies on those of the raw stages, land in any order.  What a team
    has seen before has landed, and so has all that it follows from."""
    rng = np.random.default_rng(seed)
    wrong = 0
    for _ in range(trials):
        step = int(rng.integers(0, 40))                      # the team step % teams is about to take it
        mine = range(step % teams, step, teams)              # what it has taken
        retired = int(rng.integers(max(0, max(mine, default=-1) - x + 1), step + 1))     # MMAs 0 .. retired - 1
        seen_x = {s - x for s in mine if s >= x}
        seen_raw = set(mine) | set(range(retired))           # an MMA is behind its own codes
        arrived = {s for s in range(retired) if s in seen_x or s < retired - 4 * x or rng.random() < 0.5}
        arrived |= {s for s in range(retired) if any(t % (x * sets) == s % (x * sets) and t > s for t in seen_x)}
        says = lambda done, number, ring: sum(1 for s in done if s % ring == number % ring) % 2 != number // ring % 2
        if step >= x and says(arrived, step - x, x * sets) != (step - x in arrived):
            wrong += 1
            continue
        if step >= x and step - x not in arrived:
            continue                                         # still waiting
        # X is there: every MMA up to step - x has retired
        known = max(retired, step - x + 1)
        landed = seen_raw | set(range(known)) | {s for s in range(known, known + raw) if rng.random() < 0.5}
        landed = {s for s in landed if s < known + raw}
        wrong += says(landed, step, raw) != (step in landed)
    return wrong


@pytest.mark.parametrize("which", [0, 1])
def test_model_of_the_rings(which):
    _, raw, x, teams, sets = rings()[which]
    assert model(raw, x, teams, 1 + which, sets) == 0


def test_the_model_finds_the_race():
    assert model(7, 3, 2, 3) > 0          # an X stage that two teams take in turn
    assert model(6, 8, 4, 5) > 0          # an X stage older than the raw stage
