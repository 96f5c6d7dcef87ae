"""The protocol of the places that rows pass through in pdb_distill's gradient (Stream in rows.cuh), run on the host with
barriers, copies and warps that take steps in any order: whatever waits run out, nothing is under way when the bringing
warp ends, no place is filled while its copy is under way or its barrier armed, and all ends."""
import random

import pytest


class Barrier:
    """A transaction barrier: phases of `count` arrivals and the bytes expected."""

    def __init__(self, count):
        self.count, self.phase, self.left, self.bytes = count, 0, count, 0

    def arrive(self, expect=0):
        assert self.left > 0, "an arrival too many in a phase"
        self.left -= 1
        self.bytes += expect
        self.turn()

    def complete(self, n):
        self.bytes -= n
        self.turn()

    def turn(self):
        if self.left == 0 and self.bytes == 0:
            self.phase += 1
            self.left = self.count

    def done(self, parity):
        return self.phase & 1 != parity


class Block:
    """One block: a bringing warp and its readers, each a generator that yields between its steps."""

    def __init__(self, rng, rows, chunks, slots, hold, warps, tries, bring_tries, stall):
        self.rng, self.rows, self.chunks, self.slots, self.hold = rng, rows, chunks, slots, hold
        self.warps, self.tries, self.bring_tries, self.stall = warps, tries, bring_tries, stall
        self.full = [Barrier(1) for _ in range(slots)]
        self.empty = [Barrier(warps) for _ in range(slots)]
        self.flying = []                 # slots whose copy is under way
        self.timeouts = 0
        self.at_barrier, self.generation = 0, 0
        self.stopped = False

    def wait(self, me, bar, parity):
        if bar.done(parity) or me["gave_up"]:
            return
        for _ in range(me["tries"]):
            if bar.done(parity):
                return
            yield
        me["gave_up"] = True
        self.timeouts += 1

    def sync(self):
        mine = self.generation
        self.at_barrier += 1
        if self.at_barrier == self.warps:
            self.at_barrier, self.generation = 0, mine + 1
        while self.generation == mine:
            yield

    def bring(self):
        me = {"gave_up": False, "tries": self.bring_tries}
        slot = parity = brought = 0
        passing = max(0, self.chunks - self.hold)
        for _ in range(self.rows):
            for end in (self.chunks, passing):
                for _ in range(end):
                    yield from self.wait(me, self.empty[slot], parity ^ 1)
                    if me["gave_up"]:
                        break
                    assert slot not in self.flying, "a place filled while its copy is under way"
                    self.full[slot].arrive(16)
                    self.flying.append(slot)
                    slot, parity = (0, parity ^ 1) if slot + 1 == self.slots else (slot + 1, parity)
                    brought += 1
                    yield
                if me["gave_up"]:
                    break
            if me["gave_up"]:
                break
        for _ in range(min(self.slots, brought)):
            if slot == 0:
                slot, parity = self.slots, parity ^ 1
            slot -= 1
            while not self.full[slot].done(parity):      # its limit lies far above what a copy takes
                yield
        assert not self.flying, "a copy under way when the bringing warp ends"

    def read(self, warp):
        me = {"gave_up": self.tries == 0, "tries": self.tries}
        slot = parity = 0
        passing = max(0, self.chunks - self.hold)

        def give_back(p):
            if not me["gave_up"]:
                self.empty[p].arrive()

        for _ in range(self.rows):
            yield from self.sync()
            if self.rng.random() < self.stall:
                for _ in range(self.rng.randrange(60)):
                    yield
            taken = []
            for n in range(self.chunks):
                yield from self.wait(me, self.full[slot], parity)
                taken.append(slot)
                slot, parity = (0, parity ^ 1) if slot + 1 == self.slots else (slot + 1, parity)
                yield
                if n < passing:
                    give_back(taken[-1])
            if me["gave_up"]:
                self.stopped = True
            yield from self.sync()
            yield from self.sync()
            stop = self.stopped
            for n in range(self.chunks):
                if n < self.chunks - passing:
                    p = taken[passing + n]
                else:
                    yield from self.wait(me, self.full[slot], parity)
                    p = slot
                    slot, parity = (0, parity ^ 1) if slot + 1 == self.slots else (slot + 1, parity)
                yield
                give_back(p)
            if stop:
                return

    def run(self):
        live = [self.bring()] + [self.read(w) for w in range(self.warps)]
        steps = 0
        while live:
            steps += 1
            assert steps < 2_000_000, "does not end"
            if self.flying and self.rng.random() < 0.1:
                s = self.flying.pop(self.rng.randrange(len(self.flying)))
                self.full[s].complete(16)
            g = self.rng.choice(live)
            try:
                next(g)
            except StopIteration:
                live.remove(g)


@pytest.mark.parametrize("seed", range(40))
def test_places_when_waits_run_out(seed):
    rng = random.Random(seed)
    slots = rng.randrange(3, 9)
    chunks = rng.randrange(1, 14)
    hold = max(1, min(chunks, slots - 2))
    tries = rng.choice([0, 1, 3, 10, 40])
    b = Block(rng, rng.randrange(1, 9), chunks, slots, hold, rng.choice([2, 4]), tries, tries + rng.choice([0, 5, 50]), 0.3)
    b.run()


@pytest.mark.parametrize("seed", range(10))
def test_places_when_no_wait_runs_out(seed):
    rng = random.Random(1000 + seed)
    slots = rng.randrange(3, 9)
    chunks = rng.randrange(1, 14)
    b = Block(rng, 8, chunks, slots, max(1, min(chunks, slots - 2)), 4, 10 ** 6, 10 ** 6, 0.2)
    b.run()
    assert b.timeouts == 0 and not b.stopped


def test_without_a_try_every_reader_stops_after_one_row():
    b = Block(random.Random(5), 6, 5, 4, 2, 4, 0, 30, 0.0)
    b.run()
    assert b.stopped and b.timeouts == 1          # the bringing warp's, after the places it found free
