"""What the roles of attention over a cache in 8 bits do after a wait has expired, without a GPU.

Any wait on an mbarrier may give up; from then on each other one ends or gives up, as its warp finds
the phase over or the abort flag set first.  The barriers among warps (bar.sync, barrier.red) have no limit, so
every warp that others meet there has to come: every role ends, whatever the others did.
"""

import random
import re

import pytest
from test_attend_fp8_waits_host import SHAPES, SOURCE, Cta, some_pieces

SOURCE_TEXT = SOURCE.read_text()
QUERIES = SOURCE_TEXT[SOURCE_TEXT.index("// ---- queries:"):SOURCE_TEXT.index("// ---- softmax:")]
AGREEMENT = "all_of_queries<kQueries>(ok)"  # a meeting with one outcome, in front of the loop's end


def query_meetings():
    """Meetings of the query warps in the order of the source, relative to the end of the loop after an expired wait."""
    wait, end = QUERIES.index("warp_wait_quick(&ct.q_empty"), QUERIES.index("if (!ok) break;")
    assert wait < end
    agree = QUERIES[wait:end].count(AGREEMENT)
    later = len(re.findall(r"named_barrier<|all_of_queries<", QUERIES[end:]))
    return agree, later


class Meeting:
    def __init__(self, count):
        self.count, self.said, self.outcomes = count, [], []

    def say(self, what):
        self.said.append(what)
        if len(self.said) == self.count:
            self.outcomes.append(self.said)
            self.said = []


class Expiring(Cta):
    """Roles yield ("wait", barrier, phase), answered by whether it ended, or ("meet", name, what), answered by what all said."""

    def __init__(self, *args):
        super().__init__(*args)
        self.agree, self.later = query_meetings() if self.queries > 1 else (0, 0)
        self.meetings = {f"group{h}": Meeting(4) for h in range(self.groups)}
        self.meetings["queries"] = Meeting(self.queries)

    def copies(self, r):
        for wait in super().copies(r):
            if not (yield ("wait", *wait)):
                return

    def products(self, does_scores, does_values):
        for wait in super().products(does_scores, does_values):
            if not (yield ("wait", *wait)):
                return  # the last commit's wait ends by itself, or by its limit

    def query(self):
        n = 0
        for nt, _, _ in [*self.pieces, (1, None, None)]:
            if not nt:
                continue
            ok = yield ("wait", f"q_empty{n & 1}", (n >> 1) - 1)
            for _ in range(self.agree):
                ok = all((yield ("meet", "queries", ok)))
            if not ok:
                return
            if n < sum(p[0] > 0 for p in self.pieces):
                for _ in range(self.later):
                    yield ("meet", "queries", True)
            self.bars[f"q_full{n & 1}"].arrive()
            n += 1

    def softmax(self, h, warp):
        state = {"ok": True}

        def wait(name, phase):
            if state["ok"]:
                state["ok"] = yield ("wait", name, phase)

        def meet(what):
            return any((yield ("meet", f"group{h}", what)))

        tiles = n = 0
        for nt, clears, raises in [*self.pieces, (-1, (), ())]:
            if nt == 0:
                continue
            yield from wait(f"q_full{n & 1}", n >> 1)
            if (yield from meet(not state["ok"] or nt < 0)):
                return
            for j in range(nt):
                g = tiles + j
                yield from wait(f"s_full{g & 1}", g >> 1)
                if j in clears and h == 0:
                    yield from wait(f"full1_{g % self.rings[1]}", g // self.rings[1])
                yield from meet(False)
                if j and (j, h) in raises:
                    yield from meet(False)
                    yield from wait(f"pv_done{g - 1 & 1}", g - 1 >> 1)
                self.bars[f"p_full{g & 1}"].arrive()
            tiles += nt
            for _ in range(2):
                yield from meet(False)
            yield from wait(f"pv_done{tiles - 1 & 1}", tiles - 1 >> 1)
            self.bars[f"q_empty{n & 1}"].arrive()
            n += 1

    def run(self, rng, expires):
        """`expires`: the step at which some wait gives up."""
        roles = {"copy k": self.copies(0), "copy v": self.copies(1)} | {f"query {q}": self.query() for q in range(self.queries)}
        roles |= {"scores": self.products(True, False), "values": self.products(False, True)} if self.two else {"products": self.products(True, True)}
        roles |= {f"softmax {h}.{w}": self.softmax(h, w) for h in range(self.groups) for w in range(4)}
        asks, seen, aborted, step = {}, {n: 0 for n in self.meetings}, False, 0
        places = {}

        def go(name, answer):
            try:
                ask = roles[name].send(answer)
            except StopIteration:
                asks.pop(name, None)
                return
            asks[name] = ask
            if ask[0] == "meet":
                m = self.meetings[ask[1]]
                places[name] = len(m.outcomes)
                m.say(ask[2])

        for name in roles:
            go(name, None)
        while asks:
            step += 1
            can = []
            for name, (kind, *rest) in asks.items():
                if kind == "meet":
                    if len(self.meetings[rest[0]].outcomes) > places[name]:
                        can.append((name, self.meetings[rest[0]].outcomes[places[name]]))
                else:
                    over = self.bars[rest[0]].phase > rest[1]
                    # a warp finds the phase over, or gives up: by its limit, or because another did
                    if over:
                        can.append((name, True))
                    if aborted or step == expires:
                        can.append((name, False))
            flights = [f for f, items in self.flight.items() if items]
            if not can and not flights:
                if not aborted:
                    aborted = True  # what nobody ends any more expires
                    continue
                raise AssertionError(f"these never end: {asks}")
            who = rng.choice([*can, *flights])
            if isinstance(who, str):
                items = self.flight[who]
                self.bars[items.pop(rng.randrange(len(items)) if who == "copy" else 0)].arrive()
            else:
                aborted = aborted or who[1] is False
                go(*who)
        return aborted


@pytest.mark.parametrize("shape", SHAPES)
def test_every_role_ends(shape):
    expired = 0
    for seed in range(400):
        rng = random.Random(seed)
        x = Expiring(some_pieces(rng, SHAPES[shape][0]), *SHAPES[shape])
        expired += x.run(rng, rng.randint(1, 400))
    assert expired > 100


def test_without_an_expiry_nothing_is_given_up():
    for shape in SHAPES.values():
        for seed in range(20):
            rng = random.Random(seed)
            assert not Expiring(some_pieces(rng, shape[0]), *shape).run(rng, -1)
