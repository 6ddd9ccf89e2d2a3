"""A model of the stage hand-offs of the tensor-core product (matmul_tc.cu) for packed weights: a loader, two expansion
groups that take stages by turns, and the MMAs, over mbarriers that tell phases apart by parity alone.  Copies land in any
order.  Every role has to touch a stage only for the use that it means, whatever the schedule.

The model also shows why a group looks at a stage's `empty` barrier first: without that look some schedules let a group
take the previous use of a stage, still in flight, for its own (an odd number of stages)."""
import random

import pytest


class Barrier:
    """An mbarrier: completed phases; a wait for parity p passes when the current phase's parity is not p."""

    def __init__(self, count):
        self.count, self.pending, self.phase = count, count, 0

    def arrive(self):
        assert self.pending > 0, "more arrivals than the phase takes"
        self.pending -= 1
        if self.pending == 0:
            self.pending, self.phase = self.count, self.phase + 1

    def passes(self, parity):
        return (self.phase & 1) != parity


def run(stages, uses, look, rng):
    """Runs one random schedule; returns False if a role took a stage for the wrong use."""
    full = [Barrier(1) for _ in range(stages)]
    ready = [Barrier(1) for _ in range(stages)]
    empty = [Barrier(1) for _ in range(stages)]
    holds = [None] * stages      # use whose data the raw stage holds
    expanded = [None] * stages   # use whose codes the operand holds
    flying = []                  # copies in flight
    at = {"load": 0, "g0": 0, "g1": 1, "mma": 0}

    def step(role):
        n = at[role]
        if n >= uses:
            return True
        st, parity = n % stages, (n // stages) & 1
        if role == "load":
            if empty[st].passes(parity ^ 1):
                flying.append(n)
                at[role] += 1
        elif role == "mma":
            if ready[st].passes(parity):
                if expanded[st] != n:
                    return False
                empty[st].arrive()
                at[role] += 1
        elif (not look or empty[st].passes(parity ^ 1)) and full[st].passes(parity):
            if holds[st] != n:
                return False
            expanded[st] = n
            ready[st].arrive()
            at[role] += 2
        return True

    idle = 0
    while min(at.values()) < uses:
        before = dict(at), len(flying)
        what = rng.choice(["load", "g0", "g1", "mma", "land"])
        if what == "land":
            if flying:
                n = flying.pop(rng.randrange(len(flying)))
                holds[n % stages] = n
                full[n % stages].arrive()
        elif not step(what):
            return False
        idle = idle + 1 if (dict(at), len(flying)) == before else 0
        assert idle < 2000, "the schedule came to a halt"
    return True


@pytest.mark.parametrize("stages", [2, 3, 4, 5, 6, 7, 8])
def test_every_schedule_keeps_uses_apart(stages):
    rng = random.Random(stages)
    for _ in range(300):
        assert run(stages, 60, True, rng)


@pytest.mark.parametrize("stages", [3, 5, 7])
def test_without_the_look_some_schedule_mixes_uses(stages):
    rng = random.Random(stages)
    assert not all(run(stages, 60, False, rng) for _ in range(300))
