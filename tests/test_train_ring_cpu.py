"""Layer norm's ring of copies on the CPU.  When a wait runs out, as a model: who arms a barrier and issues copies
when, with copies that land late or never; and what the copies reach."""
import os
import random
import shutil
import subprocess
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parent.parent


class Cta:
    """Warps that wait for a stage, read it and meet at a barrier, after which the first one fills it again.
    A barrier of count 1 is armed by a fill, and its phase ends when the fill's copy has landed."""

    def __init__(self, rng, stages, rounds, warps, limit, delays, stops):
        self.__dict__.update(rng=rng, stages=stages, rounds=rounds, warps=warps, limit=limit, delays=delays, stops=stops)
        self.now, self.dead, self.filled = 0, False, 0
        self.phases, self.copies = [0] * stages, {}  # phases that are over; by stage: when issued, when it lands
        self.armed_again = 0

    def tick(self):
        self.now += 1
        for stage, (_, lands) in list(self.copies.items()):
            if lands is not None and lands <= self.now:
                del self.copies[stage]
                self.phases[stage] += 1

    def wait(self, stage, parity):
        """As the kernels' bounded wait: over if the phase under way is of the other parity."""
        for _ in range(self.limit):
            self.tick()
            if self.phases[stage] % 2 != parity:
                return
            if self.dead:
                return
        self.dead = True

    def fetch(self, stage):
        if self.stops and self.dead:
            return
        self.armed_again += stage in self.copies  # armed in a phase that is not over, a copy over another
        delay = self.delays[self.filled]
        self.copies[stage] = (self.now, None if delay is None else self.now + delay)
        self.filled += 1

    def run(self):
        for s in range(min(self.stages, self.rounds)):
            self.fetch(s)
        stage = parity = 0
        for r in range(self.rounds):
            for _ in range(self.warps):
                self.wait(stage, parity)
            self.tick()  # the barrier
            if r + self.stages < self.rounds:
                self.fetch(stage)
            stage += 1
            if stage == self.stages:
                stage, parity = 0, 1 - parity
        # how long the copies that are still on their way have had
        return [self.now - issued for issued, _ in self.copies.values()]


def _all(stops):
    died = armed_again = 0
    least = None
    for seed in range(1500):
        rng = random.Random(seed)
        rounds, limit = rng.randint(1, 40), rng.randint(20, 200)
        delays = [rng.randint(1, 9) for _ in range(rounds)]
        kind = rng.randrange(4)  # all in time; some late; one late; one never
        if kind == 1:
            delays = [d if rng.random() < 0.8 else rng.randint(1, 3) * limit for d in delays]
        elif kind > 1:
            delays[rng.randrange(rounds)] = 5 * limit if kind == 2 else None
        cta = Cta(rng, rng.randint(1, 8), rounds, rng.randint(1, 16), limit, delays, stops)
        for age in cta.run():
            least = min(age - limit, least) if least is not None else age - limit
        assert not (kind == 0 and (cta.dead or cta.filled < rounds))
        died, armed_again = died + cta.dead, armed_again + cta.armed_again
    return died, armed_again, least


def test_a_wait_that_runs_out():
    died, armed_again, least = _all(True)
    assert died > 500 and armed_again == 0
    assert least >= 0  # what has not landed at the end has had the wait's whole limit
    # the model tells: going on, the first warp arms barriers twice, and leaves copies that it has just issued
    died, armed_again, least = _all(False)
    assert died > 500 and armed_again > 0 and least < 0


def test_copies_of_rows_off_16_byte_boundaries_stay_within_the_matrix(tmp_path):
    """By the kernels' own arithmetic (csrc/tula_ring.h), compiled for the host."""
    cxx = os.environ.get("CXX") or shutil.which("g++") or shutil.which("c++")
    if not cxx:
        pytest.skip("no C++ compiler")
    out = tmp_path / "ranges"
    subprocess.run([cxx, "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", "-I", str(ROOT / "paper_2603_18112_gb300" / "csrc"),
                    str(ROOT / "tests" / "ring_ranges.cpp"), "-o", str(out)], check=True)
    copies, outside = map(int, subprocess.run([str(out)], check=True, capture_output=True, text=True, timeout=120).stdout.split())
    assert copies > 100000 and outside == 0
