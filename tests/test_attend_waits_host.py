"""The barriers of attention on tensor cores, without a GPU.

A wait on an mbarrier is by parity, so it is right only while the barrier is at most one
phase ahead of its waiter: two ahead look like none.  Here the roles of a CTA (the copies
of K and of V and Q, the products and the softmax of two streams) are written down
with their waits and arrivals, in the order of csrc/serve/attend_tc.cu, and run
under random schedules in which any role, copy or commit may be held up for as long as
another one can go on.  A barrier that passes a waiter by two phases, and a state in which
nobody can go on, fail.
"""

import random
import re
from pathlib import Path

import pytest

SOURCE = Path(__file__).resolve().parent.parent / "paper_2608_29748_gb300" / "csrc" / "serve" / "attend_tc.cu"
RING_K, RING_V = {64: 5, 128: 2}, {64: 5, 128: 3}


class Lapped(AssertionError):
    pass


class Barrier:
    def __init__(self, name, count):
        self.name, self.count, self.arrived, self.phase = name, count, 0, 0

    def arrive(self):
        self.arrived += 1
        if self.arrived == self.count:
            self.arrived, self.phase = 0, self.phase + 1


class Cta:
    def __init__(self, pieces, dp, own_o_barrier):
        self.pieces, self.dp, self.own = pieces, dp, own_o_barrier
        self.bars = {}
        for r, slots in (("k", RING_K[dp]), ("v", RING_V[dp])):
            for i in range(slots):
                for c in range(3):
                    self.add(f"{r}_full{c}_{i}", 1)
                self.add(f"{r}_empty_{i}", 2)
        for s in range(2):
            for name, count in (("q_full", 1), ("q_empty", 2), ("s_full", 1), ("p_full", 4), ("o_full", 1), ("issued", 1)):
                self.add(f"{name}{s}", count)
        for s in range(2):  # bar.sync of a stream, and of both
            self.add(f"stream{s}", 4)
        self.add("both", 8)
        self.flight = {"k": [], "v": [], "q": [], "products0": [], "products1": []}  # what completes later

    def add(self, name, count):
        self.bars[name] = Barrier(name, count)

    def commit(self, s, name):
        self.flight[f"products{s}"].append(name)

    # A role yields (barrier, phase) to wait for the end of that phase; in between it arrives.
    def copies(self, ring):
        slots = (RING_K if ring == "k" else RING_V)[self.dp]
        slot = use = 0
        used, turn = [0, 0], 0
        for nt, two, _ in self.pieces:
            if nt == 0:
                continue
            if ring == "v":
                for q in range(2):
                    if not two and q != turn:
                        continue
                    yield f"q_empty{q}", used[q] - 1
                    used[q] += 1
                    self.flight["q"].append(f"q_full{q}")
                if not two:
                    turn ^= 1
            for k in range(nt):
                yield f"{ring}_empty_{slot}", use - 1
                if not two:
                    self.bars[f"{ring}_empty_{slot}"].arrive()
                self.flight[ring].append(f"{ring}_full{2 if two else k & 1}_{slot}")
                slot += 1
                if slot == slots:
                    slot, use = 0, use + 1

    def products(self, s):
        rk, rv = RING_K[self.dp], RING_V[self.dp]
        tiles = np_ = turn = batches = 0
        used, seen = [0, 0], {}

        def tile(ring, slot, two):
            name = f"{ring}_full{2 if two else s}_{slot}"
            seen[name] = seen.get(name, -1) + 1
            return name, seen[name]

        for nt, two, edges in self.pieces:
            if nt == 0:
                continue
            q, step, first = (s, 1, 0) if two else (turn, 2, s)
            yield f"q_full{q}", used[q]
            used[q] += 1
            if two:
                yield f"q_full{q ^ 1}", used[q ^ 1]
                used[q ^ 1] += 1
                self.bars[f"q_empty{q ^ 1}"].arrive()
            else:
                turn ^= 1
            j, landed = first, False
            while j < nt:
                k, v, before = (tiles + j) % rk, (tiles + j) % rv, (tiles + j - step) % rv
                yield tile("k", k, two)
                if j > first and not landed:
                    yield tile("v", before, two)
                if two and (s == 1 or batches > 0):
                    yield f"issued{s ^ 1}", batches if s == 1 else batches - 1
                if j > first:
                    yield f"p_full{s}", np_
                    np_ += 1
                    self.commit(s, f"v_empty_{before}")
                landed = j in edges
                if landed:
                    yield tile("v", v, two)
                if two:
                    self.bars[f"issued{s}"].arrive()
                    batches += 1
                self.commit(s, f"s_full{s}")
                self.commit(s, f"k_empty_{k}")
                j += step
            if j > first:
                self.commit(s, f"q_empty{q}")
                before = (tiles + j - step) % rv
                if not landed:
                    yield tile("v", before, two)
                yield f"p_full{s}", np_
                np_ += 1
                self.commit(s, f"v_empty_{before}")
                self.commit(s, f"o_full{s}" if self.own else f"s_full{s}")
            else:
                self.bars[f"q_empty{q}"].arrive()
            tiles += nt

    def softmax(self, s, warp):
        ns = no = meets = both = 0
        for nt, two, _ in self.pieces:
            self.bars[f"stream{s}"].arrive()
            yield f"stream{s}", meets
            meets += 1
            if nt == 0:
                continue
            done = 0
            for _ in range(0 if two else s, nt, 1 if two else 2):
                yield f"s_full{s}", ns
                ns += 1
                done += 1
                self.bars[f"p_full{s}"].arrive()
            if done:
                if self.own:
                    yield f"o_full{s}", no
                    no += 1
                else:
                    yield f"s_full{s}", ns
                    ns += 1
            if not two:
                for _ in range(2):
                    self.bars["both"].arrive()
                    yield "both", both
                    both += 1

    def run(self, rng):
        roles = {"copy k": self.copies("k"), "copy v": self.copies("v")}
        for s in range(2):
            roles[f"products {s}"] = self.products(s)
            for w in range(4):
                roles[f"softmax {s}.{w}"] = self.softmax(s, w)
        waits = {name: next(role, None) for name, role in roles.items()}
        held, left = None, 0
        while True:
            for name, w in waits.items():
                if w and self.bars[w[0]].phase > w[1] + 1:
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
                self.bars[items.pop(0 if who.startswith("products") else rng.randrange(len(items)))].arrive()
            else:
                waits[who] = next(roles[who], None)


def some_pieces(rng):
    pieces = []
    for _ in range(rng.randint(1, 7)):
        nt = rng.choice([0, 1, 1, 2, 3, rng.randint(1, 9)])
        pieces.append((nt, rng.random() < 0.4, {j for j in range(nt) if rng.random() < 0.3}))
    return pieces


@pytest.mark.parametrize("dp", [64, 128])
def test_no_waiter_is_lapped(dp):
    for seed in range(1500):
        rng = random.Random(seed)
        Cta(some_pieces(rng), dp, True).run(rng)


@pytest.mark.parametrize("dp", [64, 128])
def test_one_barrier_for_scores_and_the_finished_output_is_lapped(dp):
    """The order of events that the barriers of their own rule out."""
    with pytest.raises(Lapped, match="s_full"):
        for seed in range(1500):
            rng = random.Random(seed)
            Cta(some_pieces(rng), dp, False).run(rng)


def test_the_kernel_keeps_them_apart():
    """The finished output is committed to, and waited for on, o_full; scores on s_full."""
    source = SOURCE.read_text()
    assert re.findall(r"commit\(&ct\.(\w_full)\[", source) == ["s_full", "o_full"]
    assert re.findall(r"wait\(&ct\.(\w_full)\[s\], (\w+)\+\+", source) == [("p_full", "np"), ("p_full", "np"), ("s_full", "ns"), ("o_full", "no")]
