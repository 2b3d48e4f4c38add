"""Tiles with values in very different units, in the waits of attention over a cache in 8 bits, without a GPU.

A group begins such a tile as any other, agrees that it needs care, and begins it again: it waits for
the same scores once more, for the tile's values whatever the group, and meets twice for every four keys that are not
in the product.  The softmax warps agree by one word that one of them writes, so that they meet equally often even
where, after an expired wait, they have read different units.
"""

import random

import pytest
from test_attend_fp8_expiry_host import Expiring
from test_attend_fp8_waits_host import SHAPES, SOURCE, Cta, some_pieces


class Careful(Cta):
    """No wait expires: the order of csrc/serve/attend_fp8_tc.cu, with care from some tile of a piece on."""

    def __init__(self, pieces, *shape, care):
        super().__init__(pieces, *shape)
        self.care = care  # for each piece the first tile that needs care, and those that have keys apart

    def softmax(self, h, warp):
        tiles = n = meets = 0

        def meet():
            nonlocal meets
            self.bars[f"group{h}"].arrive()
            meets += 1
            return f"group{h}", meets - 1

        for (nt, clears, raises), (since, apart) in zip(self.pieces, self.care):
            if nt == 0:
                continue
            yield f"q_full{n & 1}", n >> 1
            yield meet()
            j, care = 0, False
            while j < nt:
                g = tiles + j
                yield f"s_full{g & 1}", g >> 1
                assert self.units[g % self.info] == g, "the tile's units are another's"
                if (j in clears and h == 0) or (care and j in apart):
                    yield f"full1_{g % self.rings[1]}", g // self.rings[1]
                if j:
                    yield meet()
                if j == since and not care:
                    yield meet()
                    yield meet()
                    care = True
                    continue
                if j == 0 or (j, h) in raises or (care and j in apart):
                    for _ in range(3):
                        yield meet()
                    if j:
                        yield f"pv_done{g - 1 & 1}", g - 1 >> 1
                if care and j in apart:
                    for _ in range(4):
                        yield meet()
                    assert self.units[g % self.info] == g, "the tile's units are another's"
                self.bars[f"p_full{g & 1}"].arrive()
                j += 1
            tiles += nt
            for _ in range(2):
                yield meet()
            yield f"pv_done{tiles - 1 & 1}", tiles - 1 >> 1
            self.bars[f"q_empty{n & 1}"].arrive()
            n += 1
        yield f"q_full{n & 1}", n >> 1
        yield meet()


def some_care(rng, pieces):
    return [(rng.choice([-1, rng.randrange(nt)]) if nt else -1, {j for j in range(nt) if rng.random() < 0.4}) for nt, _, _ in pieces]


@pytest.mark.parametrize("shape", SHAPES)
def test_every_wait_is_for_its_phase(shape):
    for seed in range(200):
        rng = random.Random(seed)
        pieces = some_pieces(rng, SHAPES[shape][0])
        Careful(pieces, *SHAPES[shape], care=some_care(rng, pieces)).run(rng)


class CarefulExpiring(Expiring):
    """Any wait may expire; from then on a warp sees any units."""

    def __init__(self, pieces, *shape, care, rng):
        super().__init__(pieces, *shape)
        self.care, self.rng, self.word, self.read = care, rng, {}, {}

    def softmax(self, h, warp):
        state = {"ok": True, "meets": 0}

        def wait(name, phase):
            if state["ok"]:
                state["ok"] = yield ("wait", name, phase)

        def meet(what=False):
            state["meets"] += 1
            return any((yield ("meet", f"group{h}", what)))

        def agreed():
            """The word, which all warps of the group read alike between the same two meetings."""
            return self.read.setdefault((h, state["meets"]), self.word[h])

        def agreed_and_same():
            word = agreed()
            assert word == self.word[h], "written again before all have read it"
            return word

        saw = lambda x: x if state["ok"] else self.rng.choice([False, True])  # noqa: E731
        tiles = n = 0
        for (nt, clears, raises), (since, apart) in [*zip(self.pieces, self.care), ((-1, (), ()), (-1, ()))]:
            if nt == 0:
                continue
            yield from wait(f"q_full{n & 1}", n >> 1)
            if (yield from meet(not state["ok"] or nt < 0)):
                return
            j, care = 0, False
            while j < nt:
                g = tiles + j
                yield from wait(f"s_full{g & 1}", g >> 1)
                wide, others = saw(j == since), saw(j in apart)
                if (j in clears and h == 0) or (care and others):
                    yield from wait(f"full1_{g % self.rings[1]}", g // self.rings[1])
                some, up = False, j == 0
                if j:
                    up = yield from meet(saw((j, h) in raises) or (others if care else wide))
                if up:
                    if warp == 0:
                        self.word[h] = others if care else wide
                    yield from meet()
                    some = agreed_and_same()
                    if not care and some:
                        yield from meet()
                        care = True
                        continue
                    while (yield from meet(saw(False))):
                        yield from meet()
                    yield from meet()
                    if j:
                        yield from wait(f"pv_done{g - 1 & 1}", g - 1 >> 1)
                if care and some:
                    for _ in range(4):
                        yield from meet()
                self.bars[f"p_full{g & 1}"].arrive()
                j += 1
            tiles += nt
            for _ in range(2):
                yield from meet()
            yield from wait(f"pv_done{tiles - 1 & 1}", tiles - 1 >> 1)
            self.bars[f"q_empty{n & 1}"].arrive()
            n += 1


@pytest.mark.parametrize("shape", SHAPES)
def test_every_role_ends(shape):
    for seed in range(200):
        rng = random.Random(seed)
        pieces = some_pieces(rng, SHAPES[shape][0])
        CarefulExpiring(pieces, *SHAPES[shape], care=some_care(rng, pieces), rng=rng).run(rng, rng.choice([-1, rng.randint(1, 400)]))


def test_the_kernel_agrees_by_one_word():
    source = SOURCE.read_text()
    begin, end = source.index("// ---- softmax:"), source.index("a.units[blockIdx.x] = unit;")
    softmax = source[begin:end]
    assert softmax.count("ct.others[h] =") == 1 and "if (key == 0) ct.others[h] = " in softmax
    write, meet, read = (softmax.index(x) for x in ("if (key == 0) ct.others[h] = ", "            maxima();\n            some_apart", "some_apart = ct.others[h]"))
    assert write < meet < read
    # what is done because of it depends on the word alone
    assert "if (!kCare && some_apart) {" in softmax and "if (kCare && some_apart) {" in softmax
