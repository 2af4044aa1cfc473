"""The warps of the attention kernel for chunks, played through on the CPU in any order: whoever waits for a barrier waits by a phase's parity, which tells no
more than two phases apart, so the barriers alone have to keep the warps close enough to one another, and every slot, score, probability and output has to be
what its reader takes it for, whatever the hardware schedules when.

The model has the kernel's roles (rows of both tiles, the warps that issue their contractions, fetching, the warp that sees to the values), the tensor pipe,
which does what it is given in order and late, and copies that arrive late and in any order.  The arrivals that complete a phase are taken from the kernel's
source."""
import os
import random
import re

import pytest

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2402_13720_b200", "csrc", "paged_chunk_tc.cu")
WARPS = 4                                                         # of a tile's rows


def counts():
    """Arrivals by barrier, from the kernel's source."""
    text = open(SOURCE).read()
    out = {}
    for name, n in re.findall(r"mbar_init\(&ms->(\w+)(?:\[\w+\])*, ([^)]+)\);", text):
        out[name] = {"ROW_WARPS / 2": WARPS}.get(n) or int(n)
    return out


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


class Wrong(Exception):
    pass


def play(parts, k_slots, v_slots, need, pick, p_barriers=2):
    """parts: (units of A, units of B, units) each.  pick(names): who moves next.  Returns what went wrong, or None."""
    bar = {n: [Barrier(need[n]) for _ in range(k_slots if n[0] == "k" else v_slots)] for n in ("k_full", "k_empty", "v_full", "v_ready", "v_empty")}
    q_full, s_full, s_free = ([Barrier(need[n]) for _ in range(2)] for n in ("q_full", "s_full", "s_free"))
    p_full, o_done = ([[Barrier(need[n]) for _ in range(2)] for _ in range(2)] for n in ("p_full", "o_done"))
    k, v, ready = [None] * k_slots, [None] * v_slots, [None] * v_slots
    q = [[None] * WARPS for _ in range(2)]                         # [tile][warp]: the part whose queries are there
    s = [None, None]                                               # [tile]: the unit whose scores are there
    p = [[[None] * WARPS for _ in range(2)] for _ in range(2)]
    o = [None, None]                                               # [tile]: the part, and units added up
    pipe, copies = [], []

    def expect(what, got, want):
        if got != want:
            raise Wrong(f"{what}: {got} instead of {want}")

    units = [(i, j) for i, (_, _, n) in enumerate(parts) for j in range(n)]

    def fetching():
        for u, unit in enumerate(units):
            if u >= k_slots:
                yield bar["k_empty"][u % k_slots], u // k_slots - 1
            if u >= v_slots:
                yield bar["v_empty"][u % v_slots], u // v_slots - 1
            for pool, full, n in ((k, bar["k_full"], k_slots), (v, bar["v_full"], v_slots)):
                pool[u % n] = None                                 # (from now on it may be anything)
                copies.append((pool, full, u % n, unit))
            yield None

    def values():
        for u, unit in enumerate(units):
            yield bar["v_full"][u % v_slots], u // v_slots
            expect("values to be seen to", v[u % v_slots], unit)
            ready[u % v_slots] = unit
            bar["v_ready"][u % v_slots].arrive()

    def contractions(t):
        ku = vu = scores = steps = used = 0
        for i, part in enumerate(parts):
            until, last = part[t], part[2]
            for j in range(last + 1):
                if j < last:                                       # scores of a unit
                    yield bar["k_full"][ku % k_slots], ku // k_slots
                    if j < until:
                        if j == 0:
                            yield q_full[t], used
                            used += 1
                        if scores:
                            yield s_free[t], scores - 1
                        scores += 1
                        pipe.append(("qk", t, i, j, ku % k_slots))
                        pipe.append(("done", s_full[t]))
                    pipe.append(("done", bar["k_empty"][ku % k_slots]))
                    ku += 1
                if j > 0:                                          # P V of the one before
                    yield bar["v_ready"][vu % v_slots], vu // v_slots
                    if j - 1 < until:
                        b = steps & 1
                        yield (p_full[t][b], steps >> 1) if p_barriers == 2 else (p_full[t][0], steps)
                        steps += 1
                        pipe.append(("pv", t, i, j - 1, vu % v_slots, b))
                        pipe.append(("done", o_done[t][b]))
                    pipe.append(("done", bar["v_empty"][vu % v_slots]))
                    vu += 1
                yield None

    def rows(t, w):
        steps = 0

        def bring(i):
            q[t][w] = i
            q_full[t].arrive()

        if parts[0][t]:
            bring(0)
        for i, part in enumerate(parts):
            for j in range(part[t]):
                yield s_full[t], steps
                expect("scores", s[t], (i, j))
                yield None
                expect("scores", s[t], (i, j))
                s_free[t].arrive()
                if j and random.random() < 0.3:                    # a maximum grew
                    yield o_done[t][(steps - 1) & 1], (steps - 1) >> 1
                    expect("outputs to be rescaled", o[t], (i, j))
                yield None
                p[t][steps & 1][w] = (i, j)
                p_full[t][steps & 1 if p_barriers == 2 else 0].arrive()
                steps += 1
                yield None
            if i + 1 < len(parts) and parts[i + 1][t]:
                q[t][w] = i + 1
            if part[t]:
                yield o_done[t][(steps - 1) & 1], (steps - 1) >> 1
                expect("outputs", o[t], (i, part[t]))
            if i + 1 < len(parts) and parts[i + 1][t]:
                q_full[t].arrive()
            yield None
            if part[t]:
                expect("outputs still", o[t], (i, part[t]))        # read before anything overwrites them
            yield None

    def tensor():
        while True:
            if not pipe:
                yield None
                continue
            op = pipe.pop(0)
            if op[0] == "done":
                op[1].arrive()
            elif op[0] == "qk":
                _, t, i, j, slot = op
                expect("keys", k[slot], (i, j))
                expect("queries", q[t], [i] * WARPS)
                s[t] = (i, j)
            else:
                _, t, i, j, slot, b = op
                expect("values", (v[slot], ready[slot]), ((i, j),) * 2)
                expect("probabilities", p[t][b], [(i, j)] * WARPS)
                o[t] = (i, 1) if j == 0 else (i, o[t][1] + 1)
            yield None

    def arrivals():
        while True:
            if copies:
                pool, full, slot, unit = copies.pop(random.randrange(len(copies)))
                pool[slot] = unit
                full[slot].arrive()
            yield None

    roles = {"fetching": fetching(), "values": values(), "mma a": contractions(0), "mma b": contractions(1)}
    roles.update({f"rows {t}{w}": rows(t, w) for t in range(2) for w in range(WARPS)})
    endless = {"tensor": tensor(), "copies": arrivals()}
    waits = {}
    idle = 0
    try:
        while roles:
            can = [n for n in roles if n not in waits or waits[n][0].passes(waits[n][1])] + list(endless)
            name = pick(can)
            if name in endless:
                busy = bool(pipe) if name == "tensor" else bool(copies)
                next(endless[name])
                idle = 0 if busy else idle + 1
                if idle > 200 and len(can) == 2 and not pipe and not copies:
                    return "nobody can move: " + ", ".join(sorted(roles))
                continue
            idle = 0
            waits.pop(name, None)
            try:
                x = next(roles[name])
                if x is not None:
                    waits[name] = x
            except StopIteration:
                del roles[name]
    except (Wrong, AssertionError) as e:
        return str(e) or "an arrival too many"
    return None


def some_parts(r):
    out = []
    for _ in range(r.randint(1, 6)):
        n = r.randint(1, 9)
        b = n if r.random() < 0.8 else 0
        a = n if b == 0 or r.random() < 0.5 else r.randint(0, n)
        out.append((a, b, n))
    return out


def schedules(r):
    """All alike, and with somebody far slower than the rest."""
    slow = r.choice([None, "tensor", "copies", "fetching", "values", "mma a", "mma b", "rows 0", "rows 1", "rows 00", "rows 13"])

    def pick(can):
        fast = [n for n in can if slow is None or not n.startswith(slow)]
        return r.choice(fast if fast and r.random() < 0.97 else can)

    return pick


@pytest.mark.parametrize("seed", range(60))
def test_any_schedule_is_right(seed):
    r = random.Random(seed)
    random.seed(seed)
    slots = r.choice([(4, 6), (8, 10)])
    assert play(some_parts(r), *slots, counts(), schedules(r)) is None


def test_source_has_these_barriers():
    c = counts()
    assert c["k_empty"] == c["v_empty"] == 2 and c["s_free"] == c["p_full"] == c["q_full"] == WARPS and c["v_ready"] == c["o_done"] == 1


def test_one_barrier_for_both_buffers_of_p_is_found_out():
    """The rows may be a unit ahead of P V: with one barrier for both buffers a phase is lapped, which the model has to notice."""
    found = 0
    for seed in range(60):
        r = random.Random(seed)
        random.seed(seed)
        found += play(some_parts(r), 4, 6, counts(), schedules(r), p_barriers=1) is not None
    assert found > 0


def test_an_arrival_too_few_is_found_out():
    need = counts()
    need["k_empty"] = 1                                             # A alone gives the keys back
    found = 0
    for seed in range(60):
        r = random.Random(seed)
        random.seed(seed)
        found += play(some_parts(r), 4, 6, need, schedules(r)) is not None
    assert found > 0
