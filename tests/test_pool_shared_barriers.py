"""The barriers of csrc/pool_shared.cu's shared_tiles_kernel, as a model on the CPU: its warps are agents that take their steps in any order, copies and
products are done at any time after they were issued (a stream's products in their order).  Whatever the order, every wait by parity has to
be for the phase that it means, every buffer has to hold the tile that is read from it, and nobody may wait for good."""
import os
import random
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = open(os.path.join(ROOT, "paper_2410_01699_b200", "csrc", "pool_shared.cu")).read()
K_STAGES, NOTES = (int(re.search(r"constexpr int %s = (\d+);" % name, SOURCE).group(1)) for name in ("kKStages", "kInfo"))
AHEAD = sorted(int(n) for n in re.findall(r"scores\((?:j|s\.i0) \+ (\d)\)", SOURCE))   # before a unit's first weights, beside a tile's second half, behind a tile


class Barrier:
    def __init__(self, count):
        self.count = self.pending = count
        self.phases = 0   # that are complete

    def arrive(self):
        self.pending -= 1
        assert self.pending >= 0, "arrivals of the next phase"
        if self.pending == 0:
            self.phases, self.pending = self.phases + 1, self.count

    def over(self, phase):
        """What a wait for the parity of `phase` sees."""
        over = (self.phases & 1) != (phase & 1)
        assert not over or self.phases == phase + 1, "a parity of another phase"
        return over


def simulate(units, seed, k_stages=K_STAGES, notes=NOTES, first=2, between=3, behind=3):
    """units: lists of tiles, of stream 0, of stream 1 or of both (2)."""
    rng = random.Random(seed)
    pair = lambda count: [[Barrier(count) for _ in range(2)] for _ in range(2)]
    k_full, k_empty = ([Barrier(n) for _ in range(k_stages)] for n in (1, 2))
    raw_full, raw_empty = ([Barrier(1) for _ in range(2)] for _ in range(2))
    v_full, v_empty, s_full, p_ready, o_done = pair(1), pair(2), pair(1), pair(1), pair(1)
    q_ready, q_seen, both = Barrier(2), Barrier(2), Barrier(2)   # (both: the softmax warps of the two streams meet at a unit's end)
    tiles = [kind for unit in units for kind in unit]
    copies, products = [], [[], []]   # under way
    keys, raw, values, note = [None] * k_stages, [None] * 2, [[None, None], [None, None]], [None] * notes

    def copy():
        for m in range(len(tiles)):
            if m >= k_stages:
                yield k_empty[m % k_stages], m // k_stages - 1
            note[m % notes] = m
            copies.append(("keys", m))
            if m >= 2:
                yield raw_empty[m & 1], m // 2 - 1
            copies.append(("raw", m))

    def convert():
        for m in range(len(tiles)):
            yield raw_full[m & 1], m // 2
            for half in range(2):
                if m >= 2:
                    yield v_empty[m & 1][half], m // 2 - 1
                assert raw[m & 1] == m and note[m % notes] == m
                values[m & 1][half] = m
                yield None
                assert note[m % notes] == m
                if half == 1:
                    raw_empty[m & 1].arrive()
                v_full[m & 1][half].arrive()

    def issue(stream):
        base = done = 0
        for u, unit in enumerate(units):
            yield q_ready, u
            q_seen.arrive()
            at, half_done, open_ = 0, False, [False, False]

            def scores(end):
                nonlocal at, half_done
                while at < min(end, len(unit)):
                    own, m = unit[at] in (2, stream), base + at
                    if not half_done:
                        if own and open_[0]:
                            return
                        yield k_full[m % k_stages], m // k_stages
                        assert keys[m % k_stages] == m
                        if own:
                            products[stream].append(("scores", 0, m))
                            half_done = open_[0] = True
                        else:
                            k_empty[m % k_stages].arrive()
                    if own:
                        if open_[1]:
                            return
                        products[stream] += [("scores", 1, m), ("keys", 0, m)]
                        half_done, open_[1] = False, True
                    at += 1
            yield from scores(first)
            for j, kind in enumerate(unit):
                m = base + j
                if kind in (2, stream):
                    for half in range(2):
                        yield p_ready[stream][half], done
                        yield v_full[m & 1][half], m // 2
                        products[stream] += [("out", half, m), ("values", half, m)]
                        open_[half] = False
                        if half == 0:
                            yield from scores(j + between)
                    done += 1
                else:
                    for half in range(2):
                        yield v_full[m & 1][half], m // 2
                    for half in range(2):
                        v_empty[m & 1][half].arrive()
                yield from scores(j + behind)
            base += len(unit)

    def softmax(stream):
        base = done = 0
        for u, unit in enumerate(units):
            if u:
                yield q_seen, u - 1
            q_ready.arrive()
            yield None
            mine = 0
            for j, kind in enumerate(unit):
                if kind not in (2, stream):
                    continue
                m, mine = base + j, mine + 1
                for half in range(2):
                    yield s_full[stream][half], done
                    assert note[m % notes] == m
                    yield None
                    if (mine > 1 or half) and rng.random() < 0.3:   # the reference follows a maximum: sums are multiplied
                        yield o_done[stream][1 - half], done - 1 + half
                    assert note[m % notes] == m
                    yield v_full[m & 1][half], m // 2
                    assert values[m & 1][half] == m
                    yield None
                    p_ready[stream][half].arrive()
                done += 1
            if mine:
                for half in range(2):
                    yield o_done[stream][half], done - 1
            both.arrive()
            yield both, u
            base += len(unit)

    def end_of_copy():
        what, m = copies.pop(0 if rng.random() < 0.7 else rng.randrange(len(copies)))
        buffer, full, n = (keys, k_full, k_stages) if what == "keys" else (raw, raw_full, 2)
        buffer[m % n] = m
        full[m % n].arrive()

    def end_of_product(stream):
        what, half, m = products[stream].pop(0)
        assert what != "out" or values[m & 1][half] == m
        {"scores": s_full[stream][half], "keys": k_empty[m % k_stages], "out": o_done[stream][half], "values": v_empty[m & 1][half]}[what].arrive()

    agents = {"copy": copy(), "convert": convert(), "issue 0": issue(0), "issue 1": issue(1), "softmax 0": softmax(0), "softmax 1": softmax(1)}
    waits = dict.fromkeys(agents)
    speed = {name: rng.choice((0.05, 0.3, 1, 3)) for name in (*agents, "copies", "products 0", "products 1")}
    while agents:
        ready = [name for name in agents if waits[name] is None or waits[name][0].over(waits[name][1])]
        ready += ["products %d" % stream for stream in range(2) if products[stream]] + (["copies"] if copies else [])
        assert ready, "everybody waits"
        name = rng.choices(ready, [speed[x] for x in ready])[0]
        if name == "copies":
            end_of_copy()
        elif name.startswith("products"):
            end_of_product(int(name[-1]))
        else:
            try:
                waits[name] = next(agents[name])
            except StopIteration:
                del agents[name]


def _units(rng):
    """One to three units: tiles of both streams, in turns, of both and then in turns and then of one, of one alone, of any."""
    units = []
    for _ in range(rng.randrange(1, 4)):
        n, kind = rng.randrange(1, 12), rng.randrange(5)
        if kind == 2:
            a, b, c = (rng.randrange(6) for _ in range(3))
            unit = [2] * a + [i & 1 for i in range(2 * min(b, c))] + [0 if b > c else 1] * abs(b - c)
            units.append(unit[rng.randrange(max(1, len(unit))):] or [2])
        else:
            units.append({0: [2] * n, 1: [i & 1 for i in range(n)], 3: [rng.randrange(2)] * n, 4: [rng.randrange(3) for _ in range(n)]}[kind])
    return units


def _faults(runs, **kw):
    n = 0
    for seed in range(runs):
        try:
            simulate(_units(random.Random(7 * seed + 1)), seed, **kw)
        except AssertionError:
            n += 1
    return n


def test_the_order_of_the_barriers_holds():
    assert (K_STAGES, NOTES, AHEAD) == (3, 8, [2, 3, 3])   # (what the model was made for)
    assert _faults(600) == 0


@pytest.mark.parametrize("change", [dict(between=4), dict(behind=4), dict(notes=4)])
def test_the_model_finds_what_goes_too_far(change):
    """Scores three tiles ahead of the values; too few notes."""
    assert _faults(600, **change) > 0
