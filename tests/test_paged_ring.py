"""The ring of the attention kernel for many query rows, played through on the CPU: whoever waits for a stage waits by a phase's parity, which tells
no more than two phases apart, so the barriers alone have to keep the warps within one phase of one another, whatever the hardware schedules when.

The model has the roles that meet at a stage (fetching, contractions, the warp for the units at a sequence's end) and takes the arrivals on `empty` from the
kernel's source."""
import os
import random
import re

import pytest

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2402_13720_b200", "csrc", "paged_attention_tc.cu")


class Barrier:
    def __init__(self, count):
        self.count, self.missing, self.done = count, count, 0      # done: phases completed

    def arrive(self):
        self.missing -= 1
        assert self.missing >= 0
        if self.missing == 0:
            self.missing, self.done = self.count, self.done + 1

    def passes(self, phase):                                       # what a wait for the phase's parity says
        return self.done % 2 != phase % 2


def play(stages, units, tail, empty_count, tail_arrives, pick):
    """tail[u]: unit u is at a sequence's end.  pick(names): the role that moves next.  Returns what went wrong, or None."""
    full, fixed, empty = ([Barrier(n) for _ in range(stages)] for n in (1, 1, empty_count))

    def fetching():
        for u in range(units):
            if u >= stages:
                yield empty[u % stages], u // stages - 1
            full[u % stages].arrive()

    def contractions():
        fixes = [0] * stages
        for u in range(units):
            s = u % stages
            if tail[u]:
                yield fixed[s], fixes[s]
                fixes[s] += 1
            else:
                yield full[s], u // stages
            if u:
                empty[(u - 1) % stages].arrive()                   # P V of the unit before

    def ends():
        for u in range(units):
            s = u % stages
            yield full[s], u // stages
            if tail[u]:
                fixed[s].arrive()
            if tail_arrives:
                empty[s].arrive()

    roles = {"fetching": fetching(), "contractions": contractions(), "ends": ends()}
    waits = {}

    def go_on(name):
        try:
            waits[name] = next(roles[name])
        except StopIteration:
            waits.pop(name, None)
            del roles[name]

    for name in list(roles):
        go_on(name)
    while roles:
        ready = [n for n in roles if waits[n][0].passes(waits[n][1])]
        if not ready:
            return "everybody waits"
        name = pick(ready)
        bar, phase = waits[name]
        if bar.done != phase + 1:
            return f"{name} takes phase {bar.done - 1} for {phase}"
        go_on(name)
    return None


def as_written():
    text = open(SOURCE).read()
    count = int(re.search(r"mbar_init\(&ms->empty\[i\], (\d+)\)", text).group(1))
    ends = text[text.index("units at a sequence's end\n"): text.index("================================================================ rows")]
    return count, "mbar_arrive(&ms->empty[stage])" in ends


@pytest.mark.parametrize("stages", [6, 8])
def test_no_warp_can_be_lapped_whatever_is_scheduled_when(stages):
    count, arrives = as_written()
    rng = random.Random(stages)
    for trial in range(300):
        units = rng.randrange(1, 90)
        often = rng.choice([0.0, 0.05, 0.5, 1.0])
        tail = [rng.random() < often for _ in range(units - 1)] + [True]
        late = rng.choice(["ends", "ends", "fetching", "contractions", None])     # moves only when nobody else can

        def pick(ready):
            rest = [n for n in ready if n != late]
            return rng.choice(rest or ready)

        assert play(stages, units, tail, count, arrives, pick) is None, (trial, units, late)


def test_the_model_shows_a_warp_that_nobody_waits_for():
    """The same with one arrival on `empty`, of the contractions alone."""
    late = lambda ready: next((n for n in ready if n != "ends"), "ends")
    assert play(6, 40, [False] * 39 + [True], 1, False, late) is not None
    assert play(6, 40, [False] * 39 + [True], 2, True, late) is None
