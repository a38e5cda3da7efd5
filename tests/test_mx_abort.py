"""Copies in flight when a wait of the microscaled contractions gives up: none may land after its CTA has left.

What makes that certain: a stage is released only when all of it has landed, so an issuer or a team whose wait gave up goes no further; the
producers then stop a ring behind the last release at most, each where it is; and one thread waits for what is still on its way, making up
for arrivals and bytes that a producer owes a stage which only others came to.  A wait that runs out cannot be had on
demand, so the steps are checked in the source, and the protocol in a model with barriers that count as the device's do."""
import os
import random
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2105_11010_b200", "csrc")
KERNELS = {"sparq_mxf4_small_kernel.cuh": 1, "sparq_mxf4_kernel.cuh": 1, "sparq_wgrad_kernel.cuh": 2}


def source(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


def body(text, start):
    depth, i = 0, text.index("{", start)
    for j in range(i, len(text)):
        depth += {"{": 1, "}": -1}.get(text[j], 0)
        if depth == 0:
            return text[i:j + 1]


def issuers(name):
    text = source(name)
    return [body(text, m.start()) for m in re.finditer(r"__device__ void issue\(", text)]


@pytest.mark.parametrize("name", KERNELS)
def test_no_wait_of_a_warp_is_taken_for_granted(name):
    """Every wait whose giving up would let a role go on is asked for its answer."""
    text = source(name)
    calls = [m.start() for m in re.finditer(r"\bmbar_wait_warp\(", text)]
    assert calls
    for at in calls:
        assert re.search(r"(!|= |&& |\|\| )$", text[:at]), text[at - 60:at + 60]


@pytest.mark.parametrize("name", KERNELS)
def test_an_issuer_that_gave_up_releases_nothing(name):
    found = issuers(name)
    assert len(found) == KERNELS[name]
    for src in found:
        # behind the last wait for operands: a way out, then the MMAs, then the release
        last = max(m.start() for m in re.finditer(r"mbar_wait_warp\(", src))
        release = re.search(r"tc_commit(?:_if|_pair)\(empty_bar", src).start()
        assert last < src.index("break;", last) < src.index("tc_mma_") < release
        # every MMA issued is committed to a barrier that is waited for whether or not the flag is up
        assert re.search(r"mbar_wait\(acc_bar\([^;]*, true\);", src[release:])


def test_a_team_that_gave_up_hands_nothing_on():
    text = source("sparq_wgrad_kernel.cuh")
    waits = re.findall(r"if \((?:it|stage) >= kX && !mbar_wait_warp\([^;]*x_empty_bar[^;]*\)\) return;\s*if \(!mbar_wait_warp\([^;]*raw_bar[^;]*\)\) return;\s*transform_stage\(", text)
    assert len(waits) == 2


def test_what_is_on_its_way_is_waited_for():
    small, pair, wgrad, common = (source(f) for f in ("sparq_mxf4_small_kernel.cuh", "sparq_mxf4_kernel.cuh", "sparq_wgrad_kernel.cuh", "sparq_mx_tc.cuh"))
    assert "if (!live && lane == 0) drain_two(full_bar(0), (uint32_t)S, issued," in issuers("sparq_mxf4_small_kernel.cuh")[0]
    assert "issued[LANES ? 0 : 1] = (uint32_t)it;" in small and "issued[0] = issued[1] = kStillIssuing;" in small
    for src, more in ((issuers("sparq_mxf4_kernel.cuh")[0], "2 * kHalf, 3 * T * kScaleTile"), (issuers("sparq_wgrad_kernel.cuh")[1], "2 * kWgBox, X16 ? 2 * kWgBox : 0")):
        tail = src[src.index("if (!live && lane == 0) {"):]
        assert tail.index("store_remote(map_to_rank(smem_u32((const void *)abort_flag), 1), 1u);") < tail.index("drain_pair(full_bar(0), kStages, issued, " + more)
    assert "issued + 2 * rank + (CODES ? 0 : 1))), 0), n);" in pair and "for (int q = 0; q < 4; ++q) issued[q] = kStillIssuing;" in pair
    assert "if (DY || X16) store_remote(map_to_rank(smem_u32((const void *)(issued + 2 * rank + (DY ? 0 : 1))), 0), done);" in wgrad
    # barriers of one producer's own: behind the barrier at which all roles have ended, before the CTA leaves
    assert "{ issued[DY ? 0 : 1] = (uint32_t)it; break; }" in wgrad and "issued[0] = issued[1] = (uint32_t)c.steps;" in wgrad
    kernel = wgrad[wgrad.index("sparq_wgrad_small_kernel(const"):wgrad.index("using WgradPairRings")]
    ended = kernel.index("__syncthreads();", kernel.index("switch (warp)"))
    assert ended < kernel.index("drain_ring_call(c.full_bar(0), WgradSmall::kRaw, issued[0]") < kernel.index("drain_ring_call(c.raw_bar(0), WgradSmall::kRaw, issued[1]") < kernel.index("cluster_arrive();")
    kernel = wgrad[wgrad.index("\nsparq_wgrad_kernel(const"):]
    assert kernel.index("cluster_wait();", kernel.index("switch (warp)")) < kernel.index("*c.abort_flag) drain_ring(c.raw_bar(0), Cta::kStages, issued[4]") < kernel.index("tcgen05.dealloc")
    assert "else issued[4] = done;" in wgrad
    # not cut short by the flag that is up
    assert re.search(r"mbar_wait\(bar \+ 8u \* \(j % S\), j / S & 1u, abort_flag, status, limit, true\)", common)
    assert re.search(r"mbar_wait\(at, j / S & 1u, abort_flag, status, limit, true\)", common)


# ---- the protocol -----------------------------------------------------------------------------------


class Barrier:
    def __init__(self, count):
        self.count, self.pending, self.tx, self.phase = count, count, 0, 0

    def step(self, arrivals=0, tx=0):
        assert arrivals <= self.pending, "more arrivals than the phase has"
        self.pending -= arrivals
        self.tx += tx
        if self.pending == 0 and self.tx == 0:
            self.phase += 1
            self.pending = self.count


class Run:
    """Producers of `bytes` each that count on one barrier a stage; announces[p]: what p's arrival expects (None: it does not arrive)."""

    def __init__(self, rng, S, steps, sizes, announces, releases_whole=True):
        self.rng, self.S, self.steps, self.sizes, self.announces, self.whole = rng, S, steps, sizes, announces, releases_whole
        self.bar = [Barrier(sum(a is not None for a in announces)) for _ in range(S)]
        self.issued, self.flying, self.released, self.stopped = [0] * len(sizes), [], 0, [False] * len(sizes)

    def issue(self, p):
        j = self.issued[p]
        if self.announces[p] is not None:
            self.bar[j % self.S].step(1, self.announces[p])
        self.flying.append((j, self.sizes[p]))
        self.issued[p] += 1

    def land(self):
        if self.flying:
            j, size = self.flying.pop(self.rng.randrange(len(self.flying)))
            self.bar[j % self.S].step(0, -size)

    def run(self):
        abort_at, aborted, done = self.rng.randrange(400), False, False
        for tick in range(4000):
            aborted = aborted or tick >= abort_at
            what = self.rng.randrange(3 + len(self.sizes))
            if what == 0 or what == 1:
                self.land()
            elif what == 2 and not done:
                full = self.bar[self.released % self.S].phase > self.released // self.S
                if self.released == self.steps or (not full and aborted and self.whole):
                    done = True
                elif full or aborted:
                    self.released += 1
            elif what >= 3 and not self.stopped[what - 3]:
                p = what - 3
                if self.issued[p] == self.steps:
                    self.stopped[p] = True
                elif self.issued[p] < self.released + self.S:
                    self.issue(p)
                elif aborted:
                    self.stopped[p] = True
            if done and all(self.stopped):
                return
        raise AssertionError("a role did not end")

    def wait(self, j):
        for _ in range(10000):
            if self.bar[j % self.S].phase > j // self.S:
                return
            self.land()
        raise AssertionError("waits in vain")

    def ring(self, n):
        for j in range(max(0, n - self.S), n):
            self.wait(j)

    def drain_two(self):
        n = max(self.issued)
        for j in range(min(self.issued), n):
            self.bar[j % self.S].step(1)
        self.ring(n)

    def drain_pair(self):
        n = max(self.issued)
        for j in range(max(0, n - self.S), n):
            on_way = sum(size for p, size in enumerate(self.sizes) if j < self.issued[p])
            owed = sum(self.sizes) - on_way
            if j >= self.issued[0]:
                self.bar[j % self.S].step(1, on_way)
            elif owed:
                self.bar[j % self.S].step(0, -owed)
            self.wait(j)


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("form", ["one", "two", "pair", "pair of two"])
def test_model(form, seed):
    rng = random.Random(seed)
    sizes, announces, drain = {
        "one": ([3], [3], lambda r: r.ring(r.issued[0])),
        "two": ([3, 5], [3, 5], Run.drain_two),
        "pair": ([3, 5, 3, 5], [16, None, None, None], Run.drain_pair),
        "pair of two": ([3, 3], [6, None], Run.drain_pair),
    }[form]
    uneven = 0
    for _ in range(300):
        r = Run(rng, rng.randrange(1, 8), rng.randrange(1, 40), sizes, announces)
        r.run()
        uneven += len(set(r.issued)) > 1
        drain(r)
        assert not r.flying
    assert uneven > 0 or form == "one"


def test_the_model_finds_stages_released_too_early():
    """The same with an issuer that goes on after a wait that gave up."""
    with pytest.raises(AssertionError):
        for seed in range(50):
            r = Run(random.Random(seed), 3, 30, [3, 5], [3, 5], releases_whole=False)
            r.run()
            r.drain_two()
            assert not r.flying
