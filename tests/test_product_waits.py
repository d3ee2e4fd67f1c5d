"""The waits of the feed-forward products' epilogue that goes by blocks (large tile, 16-bit matrices),
when they give up: what the source does there, and a model of the barriers of the saved projections'
slots."""
import os
import re

import paper_2608_27735_gb300 as ab


def block_epilogue():
    src = open(os.path.join(os.path.dirname(ab.__file__), "csrc", "ffproduct.cuh")).read()
    start = src.index("} else if constexpr (P::kBlocks) {")
    return src[start:src.index("tma_store_done();", start)]


def test_a_wait_gives_up_for_all_lanes_of_a_warp():
    """Below the waits the lanes meet at warp barriers, some of them only where the wait did not give
    up: so all lanes take one and the same decision.  (The slots' loader is a single lane.)"""
    waits = re.findall(r"(?m)^ *ok = (.*mbar_wait.*);$", block_epilogue())
    assert len(waits) == 2 and all(w.startswith("__all_sync(~0u, ok && mbar_wait(") for w in waits)


class Spent(Exception):
    """An arrival on a barrier whose phase has had all of its arrivals."""


class Barrier:
    """An mbarrier: a phase ends when its arrivals have come and no bytes are outstanding."""

    def __init__(self, count):
        self.count = self.pending = count
        self.bytes = self.phase = 0

    def arrive(self, expect=0):
        if self.pending == 0:
            raise Spent
        self.pending -= 1
        self.bytes += expect
        self._end()

    def land(self, n):
        self.bytes -= n
        self._end()

    def _end(self):
        if self.pending == 0 and self.bytes == 0:
            self.phase ^= 1
            self.pending = self.count

    def passed(self, parity):
        return self.phase != parity


SLOTS, WARPS = 3, 8


def run_slots(rng, blocks, polls, flight, arrives_after_giving_up):
    """The loader and the two groups of eight warps over `blocks` blocks, in random order: every wait gives up
    after `polls` polls, a copy lands after up to `flight` steps.  Returns how many waits gave up."""
    full, empty = [Barrier(1) for _ in range(2 * SLOTS)], [Barrier(WARPS) for _ in range(SLOTS)]
    copies, gave_up = [], []

    def wait(barrier, parity):
        for _ in range(polls):
            if barrier.passed(parity):
                return True
            yield
        gave_up.append(1)
        return False

    def loader():
        for q in range(blocks):
            if not (yield from wait(empty[q % SLOTS], q // SLOTS & 1 ^ 1)):
                return
            full[q % (2 * SLOTS)].arrive(1)
            copies.append((rng.randint(1, flight), full[q % (2 * SLOTS)]))
            yield

    meeting = [[0, 0], [0, 0]]                          # of a group: arrivals, meetings

    def meet(group):
        m = meeting[group]
        mine = m[1]
        m[0] += 1
        if m[0] == WARPS:
            m[0], m[1] = 0, mine + 1
        while m[1] == mine:
            yield

    def warp(group):
        ok = True
        for q in range(group, blocks, 2):
            if ok:
                ok = yield from wait(full[q % (2 * SLOTS)], q // (2 * SLOTS) & 1)
            if ok or arrives_after_giving_up:
                empty[q % SLOTS].arrive()
            yield
            for _ in range(2):
                yield from meet(group)

    agents = [loader()] + [warp(k % 2) for k in range(2 * WARPS)]
    while agents or copies:
        copies = [(left - 1, b) for left, b in copies]
        for left, b in copies:
            if left <= 0:
                b.land(1)
        copies = [c for c in copies if c[0] > 0]
        if agents:
            a = rng.choice(agents)
            try:
                next(a)
            except StopIteration:
                agents.remove(a)
    return len(gave_up)


def test_slots_of_saved_projections_when_waits_give_up():
    """As the source says who arrives, no barrier gets an arrival too many, however early the waits give
    up; and where nothing gives up all blocks are taken.  Arrivals of warps that gave up would be too many."""
    import random
    arrivals = re.findall(r"(?m)^ *if \((.*)\) mbar_arrive\w*\((slot_empty|empty0)", block_epilogue())
    assert len(arrivals) == 2
    careless = any("ok" not in condition for condition, _ in arrivals)
    gave_up = 0
    for seed in range(300):
        rng = random.Random(seed)
        gave_up += run_slots(rng, rng.randint(1, 40), rng.randint(1, 12), rng.choice((20, 200, 4000)), careless)
    assert gave_up > 100
    for seed in range(20):
        rng = random.Random(seed)
        assert run_slots(rng, rng.randint(1, 40), 10 ** 9, 200, careless) == 0
    spent = 0
    for seed in range(300):
        rng = random.Random(seed)
        try:
            run_slots(rng, 40, rng.randint(1, 12), 4000, True)
        except Spent:
            spent += 1
    assert spent > 0
