"""The rings through which tree attention's tiles of K and V go (attn_tree_tc.cu, attn_tree_rows.cu), as the sources have them: sizes, slots,
parities and places are read off the sources and run as a simulation of barriers whose waits know one bit of the phase, as the
hardware's do.  Every tile that somebody works on has to be the one that was meant, whole, and everything has to come to its end.
(A GPU that meets such a fault may hang.)"""
import random
import re

import pytest

from tests.test_wait_exits import code

TC, ROWS = "attn_tree_tc.cu", "attn_tree_rows.cu"
SPLIT, PAIR = 1, 2


def value(expr, **names):
    """A C expression of whole numbers (with casts, suffixes, `? :`) under these names."""
    e = re.sub(r"\(uint32_t\)|S::", "", expr)
    e = re.sub(r"\b(\d+)u\b", r"\1", e).replace("/", "//")
    while "?" in e:
        inner = re.search(r"\(([^()?]+) \? ([^()?:]+) : ([^()?:]+)\)", e)
        m = inner or re.fullmatch(r"()?(.+?) \? (.+?) : (.+)", e)
        c, a, b = m.groups()[-3:]
        e = e[:m.start()] + f"[{b}, {a}][bool({c})]" + e[m.end():]
    return int(eval(e, {"__builtins__": {"bool": bool}}, dict(names, kTrRows=0, kTrSplit=SPLIT, kTrPair=PAIR)))


def found(text, pattern, times=1):
    got = re.findall(pattern, text)
    assert len(got) == times and len(set(got)) == 1, (pattern, got)
    return got[0]


class Barrier:
    """Completes a phase when `count` have arrived and what was announced has landed."""

    def __init__(self, count=1):
        self.count = self.open = count
        self.loads = self.phase = 0

    def step(self, arrivals, loads=0):
        assert self.open >= arrivals, "more arrivals than a phase has"
        self.open -= arrivals
        self.loads += loads
        if self.open == 0 and self.loads == 0:
            self.open, self.phase = self.count, self.phase + 1

    def until(self, parity):                           # all that a wait can tell
        while (self.phase & 1) == (parity & 1):
            yield


class Ring:
    def __init__(self, slots, releases=1):
        self.full, self.empty = [Barrier() for _ in range(slots)], [Barrier(releases) for _ in range(slots)]
        self.holds, self.under_way = [None] * slots, []

    def load(self, slot, tile):
        self.full[slot].step(1, 1)
        self.holds[slot] = "a load under way"
        self.under_way.append((slot, tile))

    def land(self, load):
        self.under_way.remove(load)
        self.holds[load[0]] = load[1]
        self.full[load[0]].step(0, -1)

    def use(self, slot, tile):                         # a product takes a while
        for _ in range(3):
            assert self.holds[slot] == tile, f"slot {slot}: {self.holds[slot]} instead of {tile}"
            yield


def run(parts, ring, barriers, rng):
    """The parts' steps (generators; a wait is a step taken again) in any order, loads landing at any time, until all are done."""
    alive, idle = list(parts), 0
    state = lambda: [(b.phase, b.open, b.loads) for b in barriers + ring.full + ring.empty]
    while alive:
        for load in [x for x in ring.under_way if rng.random() < 0.1]:
            ring.land(load)
        before, part = state(), rng.choice(alive)
        for _ in range(rng.choice([1, 1, 3, 40])):
            if next(part, "done") == "done":
                alive.remove(part)
                break
        idle = 0 if ring.under_way or before != state() else idle + 1
        assert idle < 1000, "everybody waits"


# ---- more than 64 rows: two lanes, each with a tile of rows (PAIR) or with alternate key tiles (SPLIT) ---------------
def shared_place(j, is_v, nt):
    """Places in one ring for both lanes of SPLIT: K_0, K_1, V_0, K_2, V_1, ..."""
    return (2 * j + 2 if j + 1 < nt else 2 * j + 1) if is_v else max(2 * j - 1, 0)


def lanes(text, D, form, items, seed):
    """items: (key tiles, lane A's, lane B's)."""
    N = dict(D=D, F=form, kPair=form == PAIR)
    N["Q_TILES"] = value(found(text, r"Q_TILES = ([^;]+);"), **N)
    N["SLOTS"] = value(found(text, r" SLOTS = ([^;]+);"), **N)
    N["RING"] = value(found(text, r" RING = ([^;]+);"), **N)
    which, use, place = found(text, r"const int x = ([^,;]+), use = ([^,;]+), slot = ([^;]+);\n\s*wait\(kv_empty\(slot\)")
    empty_parity = found(text, r"wait\(kv_empty\(slot\), ([^;]+)\);")
    ahead = value(found(text, r"constexpr int kAhead = ([^;]+);"), **N)
    waits = [found(text, r"const int t = ([^,;]+), slot = ([^;]+);\s*wait\(kv_full\(slot\), ([^;]+)\);\s*return slot;"),
             found(text, r"const int t = ([^;]+), slot = ([^;]+);\s*mbar_wait_spin\(kv_full\(slot\), ([^;]+), abort_flag\);")]
    advance = found(text, r"ring0 \+= ([^;]+);", times=2).replace("I.nt", "nt")
    releases = value(found(text, r"mbar_init\(kv_empty\(i\), ([^)]+)\)"), **N)
    tile_of = found(text, r"int tr_tile\(int i, int x\) \{ return ([^;]+); \}")
    ring, rng = Ring(N["SLOTS"], releases), random.Random(seed)
    scores, ready = [Barrier(), Barrier()], [Barrier(), Barrier()]

    def producer():
        count = [0, 0]

        def load(item, is_v, j):
            x = value(which, j=j, **N)
            slot, parity = value(place, x=x, ring=count, **N), value(empty_parity, use=value(use, x=x, ring=count, **N))
            yield from ring.empty[slot].until(parity)
            count[x] += 1
            ring.load(slot, (item, is_v, j))
        for item, (nt, *_) in enumerate(items):
            yield from load(item, 0, 0)
            if form == SPLIT and nt > 1:
                yield from load(item, 0, 1)
            for j in range(nt):
                yield from load(item, 1, j)
                if j + ahead < nt:
                    yield from load(item, 0, j + ahead)

    def full(who, x, ring0, u, is_v, nt):
        """waits for a tile as the issuer (0) or the softmax (1) does; its slot"""
        t, slot, parity = waits[who]
        j = value(tile_of, i=u, x=x, **N)
        t = value(t, ring0=ring0, u=u, is_v=is_v, x=x, there=shared_place(j, is_v, nt), **N)
        slot = value(slot, t=t, x=x, **N)
        yield from ring.full[slot].until(value(parity, t=t, **N))
        return slot

    def issuer(x):
        ring0 = g0 = 0
        for item, (nt, *own) in enumerate(items):
            mine, tile = own[x], lambda u: value(tile_of, i=u, x=x, **N)
            for u in range(-1, mine) if mine else ():
                v = (yield from full(0, x, ring0, u, 1, nt)) if u >= 0 else None
                k = (yield from full(0, x, ring0, u + 1, 0, nt)) if u + 1 < mine else None
                if v is not None:
                    yield from ready[x].until(g0 + u)
                    yield from ring.use(v, (item, 1, tile(u)))
                    ring.empty[v].step(1)
                if k is not None:
                    yield from ring.use(k, (item, 0, tile(u + 1)))
                    scores[x].step(1)
                    ring.empty[k].step(1)
            for j in range(mine, nt) if form == PAIR else ():          # tiles that only the other lane uses
                for is_v in (0, 1):
                    ring.empty[(yield from full(0, x, ring0, j, is_v, nt))].step(1)
            ring0, g0 = ring0 + value(advance, n_sub=mine, nt=nt, **N), g0 + mine

    def softmax(x):
        ring0 = g0 = 0
        for item, (nt, *own) in enumerate(items):
            for u in range(own[x]):
                yield from scores[x].until(g0 + u)
                if value(tile_of, i=u, x=x, **N) == nt - 1:            # V's rows behind the sequence's last are cleared
                    yield from ring.use((yield from full(1, x, ring0, u, 1, nt)), (item, 1, nt - 1))
                ready[x].step(1)
            ring0, g0 = ring0 + value(advance, n_sub=own[x], nt=nt, **N), g0 + own[x]
    run([producer(), issuer(0), issuer(1), softmax(0), softmax(1)], ring, scores + ready, rng)


def shares(seed, form):
    rng = random.Random(seed)
    tiles = [rng.choice([1, 1, 2, 3, 4, 7, 20]) for _ in range(rng.randint(1, 5))]
    return [(n, (n + 1) >> 1, n >> 1) if form == SPLIT else (n, rng.choice([n, rng.randint(0, n)]), rng.choice([n, n, 0])) for n in tiles]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("form", [SPLIT, PAIR])
def test_lanes_get_the_tiles_that_are_meant(form, D):
    text = code(TC)
    assert found(text, r"else L\.n_tiles = ([^;]+);") == "(I.nt + 1 - x) >> 1"         # (as in shares)
    for seed in range(25):
        lanes(text, D, form, shares(seed, form), seed)


ONE_RING = [("RING = kPair ? SLOTS : SLOTS / 2;", "RING = SLOTS;"), ("const int x = F == kTrSplit ? j & 1 : 0, use", "const int x = 0, use"),
            ("(F == kTrSplit ? x * S::RING : 0) + t", "t"), ("t = ring0 + 2 * u + is_v", "t = ring0 + there"),
            ("t = ring0 + 2 * u + 1", "t = ring0 + there"), ("ring0 += 2 * (F == kTrSplit ? n_sub : I.nt)", "ring0 += 2 * I.nt")]


@pytest.mark.parametrize("change", [
    ONE_RING, [ONE_RING[0]], [ONE_RING[5]], [ONE_RING[1]], [("use = ring[x] / S::RING", "use = ring[x] / S::RING + 1")],
    [("kAhead = F == kTrSplit ? 2 : 1;", "kAhead = 1;")], [("t = ring0 + 2 * u + is_v", "t = ring0 + 2 * u + 1 - is_v")]])
def test_changes_to_the_lanes_rings_are_noticed(change):
    """One ring for lanes that wait for alternate tiles above all: a wait by parity takes a use of a slot for the one two uses back."""
    text = code(TC)
    for old, new in change:
        assert old in text
        text = text.replace(old, new)
    with pytest.raises((AssertionError, IndexError)):
        for seed in range(60):
            lanes(text, 128, SPLIT, [(20, 10, 10)] * 3, seed)


# ---- up to 64 rows: one ring, K a tile ahead ---------------------------------------------------------------------------
def few_rows(text, D, items, seed, buffers=2):
    """items: key tiles of each; buffers: of probabilities."""
    slots = value(found(text, r" SLOTS = ([^;]+);"), D=D)
    pos_k, pos_v = (found(text, r"auto pos_%s = \[&\]\(int g[^)]*\) \{ return ([^;]+); \};" % x) for x in "kv")
    assert re.search(r"load\(0, I\.h, entry, pages\);\s*if \(!stop && g > 0\) load\(1,.*\n(.*\n)*?.*if \(!stop && g > 0\) load\(1,", text)
    place, empty_parity = found(text, r"const int slot = (ring [^;]+);\s*wait\(kv_empty\(slot\), ([^;]+)\);")
    waits = [found(text, r"wait\(kv_full\(pos % S::SLOTS\), ([^;]+)\); return (pos [^;]+);"),
             found(text, r"slot = (pos [^;]+);\s*mbar_wait_spin\(kv_full\(slot\), ([^;]+), abort_flag\);")[::-1]]
    ring, rng, total = Ring(slots), random.Random(seed), sum(items)
    scores, free, ready, taken = ([Barrier(), Barrier()] for _ in range(4))
    ends = {sum(items[:i + 1]) - 1 for i in range(len(items))}

    def producer():
        order = [t for g in range(total) for t in ((0, g), (1, g - 1)) if t[1] >= 0] + [(1, total - 1)]
        for n, tile in enumerate(order):
            slot = value(place, ring=n, SLOTS=slots)
            yield from ring.empty[slot].until(value(empty_parity, ring=n, SLOTS=slots))
            ring.load(slot, tile)

    def full(who, pos):
        yield from ring.full[value(waits[who][1], pos=pos, SLOTS=slots)].until(value(waits[who][0], pos=pos, SLOTS=slots))
        return value(waits[who][1], pos=pos, SLOTS=slots)

    def issuer():
        for g in range(total + 1):
            if g < total:
                k = yield from full(0, value(pos_k, g=g))
                yield from free[g & 1].until((g >> 1) ^ 1)
                yield from ring.use(k, (0, g))
                scores[g & 1].step(1)
                ring.empty[k].step(1)
            if g > 0:
                v = yield from full(0, value(pos_v, g=g - 1, last=g == total))
                p = (g - 1) % buffers
                yield from ready[p].until((g - 1) // buffers)
                yield from ring.use(v, (1, g - 1))
                ring.empty[v].step(1)
                taken[p].step(1)

    def softmax():
        for g in range(total):
            yield from scores[g & 1].until(g >> 1)
            free[g & 1].step(1)
            yield from taken[g % buffers].until((g // buffers) ^ 1)
            if g in ends:
                yield from ring.use((yield from full(1, value(pos_v, g=g, last=g == total - 1))), (1, g))
            ready[g % buffers].step(1)
    run([producer(), issuer(), softmax()], ring, scores + free + ready + taken, rng)


@pytest.mark.parametrize("buffers", [1, 2])
@pytest.mark.parametrize("D", [64, 128])
def test_few_rows_get_the_tiles_that_are_meant(D, buffers):
    text = code(ROWS)
    for seed in range(40):
        rng = random.Random(seed)
        few_rows(text, D, [rng.choice([1, 1, 2, 3, 9, 20]) for _ in range(rng.randint(1, 6))], seed, buffers)


@pytest.mark.parametrize("old,new", [("last ? 2 * g + 1 : 2 * g + 2", "2 * g + 2"), ("last ? 2 * g + 1 : 2 * g + 2", "2 * g + 1"),
                                     ("g == 0 ? 0 : 2 * g - 1", "2 * g"), ("(uint32_t)(pos / S::SLOTS)", "(uint32_t)(pos / S::SLOTS + 1)")])
def test_changes_to_the_few_rows_ring_are_noticed(old, new):
    text = code(ROWS)
    assert old in text
    with pytest.raises((AssertionError, IndexError)):
        for seed in range(40):
            few_rows(text.replace(old, new), 128, [9, 3], seed)
