"""The barriers of the bf16 chunk attention (csrc/chunk_sm100.cu), as a model: loaders, MMA warps and softmax warps as steps between
waits, an mbarrier as a phase with a count, loads and products that finish whenever they like.  A parity wait cannot tell a phase from
the one two before it, so a warp that looks at a place of the V ring must know that the fill before the one it waits for has landed.  The
model says where one does not, under any order of events that a random schedule finds, and whether anything waits for good.  (A tile
used too early is wrong output, and a place refilled under a product: not to be looked for on a GPU.)"""
import os
import random
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_18753_b200", "csrc")


class Barrier:
    def __init__(self, count):
        self.count, self.left, self.phase = count, count, 0

    def arrive(self):
        self.left -= 1
        assert self.left >= 0, "more arrivals than a phase has"
        if self.left == 0:
            self.phase, self.left = self.phase + 1, self.count

    def passes(self, parity):           # try_wait.parity: the current phase is not the one of that parity
        return (self.phase & 1) != parity


class Early(Exception):
    pass


def run(pieces, rng, seen=True, slow=()):
    """pieces: (tiles, two) of a block's range in order.  seen: the MMA warps tell each other that a piece's V tiles have landed.  slow: V
    tiles that land late.  Raises Early where a V tile is used, or cleared, before it is there; AssertionError on a stand-still."""
    names = ["Q_FULL", "Q_EMPTY", "V_SEEN"] + [f"{n}{k}" for n in ("K_FULL", "K_EMPTY", "V_FULL", "V_EMPTY", "S_FULL", "P_FULL", "PV_DONE", "O_FREE") for k in (0, 1)]
    bar = {n: Barrier(2 if n == "Q_EMPTY" or n == "V_SEEN" or n[:-1] in ("K_EMPTY", "V_EMPTY") else 1) for n in names}
    ring = {"K": [None, None], "V": [None, None]}             # the tile that has landed in a place
    later = []                                                # events under way: (chain, action); of a chain the first comes first

    def load(which, tile, full):
        ring[which][tile % 2] = None
        def land():
            ring[which][tile % 2] = tile
            bar[full].arrive()
        later.append(((which, tile), land))

    def k_loader():
        cnt = 0
        for q, (n, two) in enumerate(pieces):
            if q:
                yield "Q_EMPTY", (q - 1) & 1
            later.append((("Q", q), bar["Q_FULL"].arrive))
            for _ in range(n):
                if cnt >= 2:
                    yield f"K_EMPTY{cnt % 2}", (cnt // 2 - 1) & 1
                load("K", cnt, f"K_FULL{cnt % 2}")
                cnt += 1

    def v_loader():
        for cnt in range(sum(n for n, _ in pieces)):
            if cnt >= 2:
                yield f"V_EMPTY{cnt % 2}", (cnt // 2 - 1) & 1
            load("V", cnt, f"V_FULL{cnt % 2}")

    def use(which, tile, what):
        if ring[which][tile % 2] != tile:
            raise Early(f"{what} of {which} tile {tile}: its place holds {ring[which][tile % 2]}")

    def mma(s):
        base = it = 0
        commit = lambda name: later.append((("mma", s), bar[name].arrive))  # noqa: E731
        def release(name, two):
            commit(name)
            if not two:
                commit(name)
        for q, (n, two) in enumerate(pieces):
            steps = n if two else (n + 1) // 2 if s == 0 else n // 2
            tile = lambda i: base + (i if two else 2 * i + s)  # noqa: E731, B023
            yield "Q_FULL", q & 1
            if seen and q:
                yield "V_SEEN", (q - 1) & 1
            for i in range(-1, steps):
                if i >= 0:
                    c = tile(i)
                    yield f"V_FULL{c % 2}", (c // 2) & 1
                    if seen and i + 1 == steps:
                        bar["V_SEEN"].arrive()
                    if i == 0 and q:
                        yield f"O_FREE{s}", (q - 1) & 1
                    if i + 1 < steps:
                        yield f"K_FULL{tile(i + 1) % 2}", (tile(i + 1) // 2) & 1
                    yield f"P_FULL{s}", (it + i) & 1
                    later.append((("mma", s), lambda c=c: use("V", c, "product")))
                    commit(f"PV_DONE{s}")
                    release(f"V_EMPTY{c % 2}", two)
                elif steps:
                    yield f"K_FULL{tile(0) % 2}", (tile(0) // 2) & 1
                if i + 1 < steps:
                    later.append((("mma", s), lambda c=tile(i + 1): use("K", c, "scores")))
                    commit(f"S_FULL{s}")
                    release(f"K_EMPTY{tile(i + 1) % 2}", two)
                    if i + 2 == steps:
                        commit("Q_EMPTY")
            if steps == 0:
                bar["Q_EMPTY"].arrive()
                if seen:
                    bar["V_SEEN"].arrive()
            base, it = base + n, it + steps

    def softmax(s):
        base = it = 0
        for n, two in pieces:
            steps = n if two else (n + 1) // 2 if s == 0 else n // 2
            for i in range(steps):
                c = base + (i if two else 2 * i + s)
                yield f"S_FULL{s}", (it + i) & 1
                if c + 1 == base + n:                         # the unit's tail is cleared in the tile
                    yield f"V_FULL{c % 2}", (c // 2) & 1
                    use("V", c, "clearing")
                bar[f"P_FULL{s}"].arrive()
            if steps:
                yield f"PV_DONE{s}", (it + steps - 1) & 1
            bar[f"O_FREE{s}"].arrive()
            base, it = base + n, it + steps

    actors = [k_loader(), v_loader(), mma(0), mma(1), softmax(0), softmax(1)]
    waits = {}
    for a in actors:
        waits[a] = next(a, None)
    while any(w is not None for w in waits.values()) or later:
        ready = [a for a, w in waits.items() if w is not None and bar[w[0]].passes(w[1])]
        first = {}
        for k, (chain, _) in enumerate(later):
            first.setdefault(chain, k)
        events = [k for c, k in first.items() if not (c[0] == "V" and c[1] in slow)]
        if not events and not ready:
            events = list(first.values())
        assert ready or events, ("stand-still", {w for w in waits.values() if w})
        if ready and (not events or rng.random() < 0.5):
            a = rng.choice(ready)
            waits[a] = next(a, None)
        else:
            later.pop(rng.choice(events))[1]()


LENGTHS = [[(3, False), (3, False)], [(3, False), (4, False)], [(1, False), (2, False), (5, False)], [(1, False)] * 5,
           [(5, False), (3, True), (4, False)], [(3, False), (2, True), (3, True), (1, False)], [(2, True), (1, False), (3, False), (2, False)],
           [(4, False), (2, False)], [(7, False), (1, False), (1, False), (6, False)], [(1, True), (1, False), (1, True), (3, False), (2, False)]]


@pytest.mark.parametrize("pieces", LENGTHS)
def test_no_tile_is_used_before_it_has_landed(pieces):
    rng = random.Random(str(pieces))
    tiles = sum(n for n, _ in pieces)
    for k in range(150):
        run(pieces, rng, slow={t for t in range(tiles) if rng.random() < 0.3} if k % 2 else ())


def test_random_ranges():
    rng = random.Random(0)
    for _ in range(400):
        pieces = [(rng.randint(1, 6), rng.random() < 0.4) for _ in range(rng.randint(1, 6))]
        run(pieces, rng, slow={t for t in range(40) if rng.random() < 0.3})


def test_without_word_of_the_landing_a_tile_is_used_early():
    """The fault that the word is for, planted in the model: behind an odd number of tiles in turns the places change owner."""
    rng = random.Random(1)
    for pieces, late in (([(3, False), (3, False)], 2), ([(5, False), (3, False)], 4), ([(3, False), (2, True)], 2)):
        with pytest.raises(Early):
            for _ in range(200):
                run(pieces, rng, seen=False, slow={late})
    for _ in range(200):                                       # even numbers never change owner
        run([(4, False), (2, False), (6, False)], rng, seen=False, slow={t for t in range(12) if rng.random() < 0.3})


def test_the_kernel_gives_and_awaits_the_word():
    """The model's order in the source: the MMA warps wait for the word of the piece before ahead of their first scores, and give theirs
    behind the wait for their last V tile, or at once where they have none."""
    text = open(os.path.join(CSRC, "chunk_sm100.cu")).read()
    role = text[text.index("MMA issuers: warp 10"):text.index("softmax, epilogue ====")]
    wait = role.index("wait_all(bar(V_SEEN), (q_cnt - 1) & 1)")
    assert wait < role.index("if (steps > 0) qk(0);")
    given = [m.start() for m in re.finditer(r"mbar_arrive\(bar\(V_SEEN\)\)", role)]
    assert len(given) == 2 and role.index("if (steps > 0) qk(0);") < given[0] < role.index("for (int i = 0; i < steps; ++i)")
    assert role.index("bar(V_FULL + st)") < given[1] < role.index("bar(P_FULL + 2 * s + half)")
