"""The barriers of attention over a cache in 8 bits, without a GPU.

The roles of a CTA (the copies of K and V, the queries, the products by one warp or two, the
groups of softmax warps) are written down with their waits and arrivals, in the order of
csrc/serve/attend_fp8_tc.cu, and run under random schedules in which any role, copy or commit may
be held up for as long as another one can go on.  A wait is by parity: it is right while its
barrier is in the phase that is waited for or the next one.
"""

import random
import re
from pathlib import Path

import pytest
from test_attend_waits_host import Barrier, Lapped

SOURCE = Path(__file__).resolve().parent.parent / "paper_2608_29748_gb300" / "csrc" / "serve" / "attend_fp8_tc.cu"
INFO = 16  # tiles whose units are kept


class Cta:
    def __init__(self, pieces, groups, products, queries, ring_k, ring_v, info=INFO):
        self.pieces, self.groups, self.two, self.queries, self.rings, self.info = pieces, groups, products == 2, queries, (ring_k, ring_v), info
        self.bars = {}
        for r in range(2):
            for i in range(self.rings[r]):
                self.add(f"full{r}_{i}", 1)
                self.add(f"empty{r}_{i}", 1)
        for b in range(2):
            for name, count in (("q_full", queries), ("q_empty", 1 + 4 * groups), ("s_full", 1), ("p_full", 4 * groups), ("pv_done", 1)):
                self.add(f"{name}{b}", count)
        for h in range(groups):
            self.add(f"group{h}", 4)
        self.flight = {"copy": [], "scored": [], "summed": []} if self.two else {"copy": [], "both": []}
        self.units = {}  # slot: tile

    def add(self, name, count):
        self.bars[name] = Barrier(name, count)

    def copies(self, r):
        tiles = 0
        for nt, _, _ in self.pieces:
            for _ in range(nt):
                slot, use = tiles % self.rings[r], tiles // self.rings[r]
                yield f"empty{r}_{slot}", use - 1
                if r == 0:
                    self.units[tiles % self.info] = tiles
                self.flight["copy"].append(f"full{r}_{slot}")
                tiles += 1

    def query(self):
        n = 0
        for nt, _, _ in self.pieces:
            if nt:
                yield f"q_empty{n & 1}", (n >> 1) - 1
                self.bars[f"q_full{n & 1}"].arrive()
                n += 1
        yield f"q_empty{n & 1}", (n >> 1) - 1  # the end
        self.bars[f"q_full{n & 1}"].arrive()

    def scores(self, g, flight):
        b, slot = g & 1, g % self.rings[0]
        yield f"full0_{slot}", g // self.rings[0]
        if self.two and g >= 2:
            yield f"pv_done{b}", (g >> 1) - 1
        self.flight[flight] += [f"s_full{b}", f"empty0_{slot}"]

    def values(self, g, flight):
        b, slot = g & 1, g % self.rings[1]
        yield f"full1_{slot}", g // self.rings[1]
        yield f"p_full{b}", g >> 1
        self.flight[flight] += [f"pv_done{b}", f"empty1_{slot}"]

    def products(self, does_scores, does_values):
        flight = "both" if does_scores and does_values else "scored" if does_scores else "summed"
        tiles = n = 0
        for nt, _, _ in self.pieces:
            if nt == 0:
                continue
            if does_scores:
                yield f"q_full{n & 1}", n >> 1
            if does_scores and does_values:
                for i in range(min(2, nt)):
                    yield from self.scores(tiles + i, flight)
                for i in range(nt):
                    yield from self.values(tiles + i, flight)
                    if i + 2 < nt:
                        yield from self.scores(tiles + i + 2, flight)
            else:
                for i in range(nt):
                    yield from (self.scores if does_scores else self.values)(tiles + i, flight)
            if does_scores:
                self.flight[flight].append(f"q_empty{n & 1}")
            n += 1
            tiles += nt

    def softmax(self, h, warp):
        tiles = n = meets = 0

        def meet():
            nonlocal meets
            self.bars[f"group{h}"].arrive()
            meets += 1
            return f"group{h}", meets - 1

        for nt, clears, raises in self.pieces:
            if nt == 0:
                continue
            yield f"q_full{n & 1}", n >> 1
            yield meet()
            for j in range(nt):
                g = tiles + j
                yield f"s_full{g & 1}", g >> 1
                assert self.units[g % self.info] == g, "the tile's units are another's"
                if j in clears and h == 0:
                    yield f"full1_{g % self.rings[1]}", g // self.rings[1]
                yield meet()
                if j and (j, h) in raises:
                    yield meet()
                    yield f"pv_done{g - 1 & 1}", g - 1 >> 1
                self.bars[f"p_full{g & 1}"].arrive()
            tiles += nt
            for _ in range(2):
                yield meet()
            yield f"pv_done{tiles - 1 & 1}", tiles - 1 >> 1
            self.bars[f"q_empty{n & 1}"].arrive()
            n += 1
        yield f"q_full{n & 1}", n >> 1
        yield meet()

    def run(self, rng):
        roles = {"copy k": self.copies(0), "copy v": self.copies(1)}
        for q in range(self.queries):
            roles[f"query {q}"] = self.query()
        if self.two:
            roles |= {"scores": self.products(True, False), "values": self.products(False, True)}
        else:
            roles["products"] = self.products(True, True)
        for h in range(self.groups):
            for w in range(4):
                roles[f"softmax {h}.{w}"] = self.softmax(h, w)
        waits = {name: next(role, None) for name, role in roles.items()}
        held, left = None, 0
        while True:
            for name, w in waits.items():
                if w and not w[1] <= self.bars[w[0]].phase <= w[1] + 1:
                    raise Lapped(f"{name} waits for phase {w[1]} of {w[0]}, which is at {self.bars[w[0]].phase}")
            ready = [n for n, w in waits.items() if w and self.bars[w[0]].phase == w[1] + 1]
            ready += [f for f, items in self.flight.items() if items]
            if not ready:
                assert not any(waits.values()), {n: w for n, w in waits.items() if w}
                return
            if left == 0:  # somebody else is held up for a while
                held, left = rng.choice([*roles, *self.flight]), rng.randint(0, 60)
            left -= 1
            who = rng.choice([r for r in ready if r != held] or ready)
            if who in self.flight:
                items = self.flight[who]
                # copies land in any order, commits complete in theirs
                self.bars[items.pop(rng.randrange(len(items)) if who == "copy" else 0)].arrive()
            else:
                waits[who] = next(roles[who], None)


def some_pieces(rng, groups):
    pieces = []
    for _ in range(rng.randint(1, 7)):
        nt = rng.choice([0, 1, 1, 2, 3, rng.randint(1, 9), rng.randint(1, 25)])
        pieces.append((nt, {j for j in range(nt) if rng.random() < 0.3},
                       {(j, h) for j in range(nt) for h in range(groups) if rng.random() < 0.3}))
    return pieces


SHAPES = {"few, 64": (1, 1, 1, 5, 6), "few, 128": (1, 1, 1, 2, 3), "least": (1, 1, 1, 2, 2), "rows, 64": (3, 2, 4, 8, 8), "rows, 128": (3, 2, 4, 3, 4),
          "rows, least": (3, 2, 1, 2, 2)}


@pytest.mark.parametrize("shape", SHAPES)
def test_every_wait_is_for_its_phase(shape):
    for seed in range(300):
        rng = random.Random(seed)
        Cta(some_pieces(rng, SHAPES[shape][0]), *SHAPES[shape]).run(rng)


def test_units_kept_too_short_a_time_are_found():
    with pytest.raises(AssertionError, match="units"):
        for seed in range(300):
            rng = random.Random(seed)
            Cta(some_pieces(rng, 1), *SHAPES["few, 64"], info=4).run(rng)


def test_the_kernel_has_these_waits():
    source = SOURCE.read_text()
    assert int(re.search(r"kInfoTiles = (\d+)", source)[1]) == INFO
    assert re.findall(r"tc_commit\(smem_u32\(&ct\.(\w+)\[", source) == ["s_full", "empty", "pv_done", "empty", "q_empty", "done"]
    assert re.findall(r"wait(?:_quick)?\(&ct\.(\w+)\[", source) == [
        "empty", "full", "pv_done", "full", "p_full", "q_full", "q_empty", "q_full", "s_full", "full", "pv_done", "pv_done"]
