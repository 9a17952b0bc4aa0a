"""The barriers of prompt_attn_kernel as a model on the host: who waits for what, in which order, with copies and products that
complete at any time.  A barrier tells the phase that is over by its parity, as the hardware's does, so a wait that comes a phase
early or late passes, or never does, here too."""
import os
import re

import paper_2607_19456_b200 as moa

SOURCE = os.path.join(os.path.dirname(moa.__file__), "csrc", "moa_prompt.cuh")


def source():
    """The kernel's text without comments."""
    with open(SOURCE) as f:
        return re.sub(r"//[^\n]*", "", f.read())


class Early(Exception):
    """A wait that passed before its phase was over, or data that was used, or overwritten, too early."""


class Barrier:
    def __init__(self, count):
        self.count = self.left = count
        self.over = 0                                      # phases

    def arrive(self, n=1):
        for _ in range(n):
            self.left -= 1
            if self.left == 0:
                self.left, self.over = self.count, self.over + 1

    def passes(self, phase):
        return (self.over & 1) != (phase & 1)


class Model:
    """units: (pair, tiles of slot 0, tiles of slot 1); a pair takes them by turns, else slot 0 sees the first of slot 1's.

    weights_first: of a step's number: whether an issuing warp waits there for the weights before it waits for V.
    join_waits: a slot waits for the other one's reads of the join before, ahead of writing its own share of the next."""

    def __init__(self, rng, units, stages, weights_first, join_waits):
        self.rng, self.units, self.NST = rng, units, stages
        self.weights_first, self.join_waits = weights_first, join_waits
        n = range(stages)
        self.k_full, self.v_full = [Barrier(1) for _ in n], [Barrier(1) for _ in n]
        self.k_empty, self.v_empty = [Barrier(2) for _ in n], [Barrier(2) for _ in n]
        self.s_full, self.p_full = ([[Barrier(1) for _ in "hh"] for _ in "ss"] for _ in range(2))
        self.o_full = [Barrier(1), Barrier(1)]
        self.q_full, self.q_empty = Barrier(1), Barrier(2)
        self.item_full, self.item_empty = [Barrier(1), Barrier(1)], [Barrier(4), Barrier(4)]
        self.joined, self.parted = Barrier(2), Barrier(2)
        self.v_at = [None] * stages                        # the tile that has landed there
        self.ml = [None, None]                             # the unit whose share a slot has written
        self.flying, self.queue = [], [[], []]             # copies under way; products and what is told behind them, a queue for each issuing warp

    # ---- waits
    def wait(self, barrier, phase):
        while not barrier.passes(phase):
            yield
        if barrier.over != phase + 1:
            raise Early("passed for phase %d with %d over" % (phase, barrier.over))
        yield

    def steps(self, unit, s):
        return unit[1 + s]

    def tiles(self, unit):
        return unit[1] + unit[2] if unit[0] else unit[2]

    # ---- who does what
    def copies(self):
        nk = nq = 0
        for n, unit in enumerate(self.units + [None]):
            if n >= 2:
                yield from self.wait(self.item_empty[n & 1], (n >> 1) - 1)
            self.item_full[n & 1].arrive()
            if unit is None:
                return
            for t in range(self.tiles(unit)):
                st = nk % self.NST
                if nk >= self.NST:
                    yield from self.wait(self.k_empty[st], nk // self.NST - 1)
                self.flying.append((self.k_full[st], None, None))
                if t == 0:
                    if nq > 0:
                        yield from self.wait(self.q_empty, nq - 1)
                    nq += 1
                    self.q_full.arrive()
                if nk >= self.NST:
                    yield from self.wait(self.v_empty[st], nk // self.NST - 1)
                if not unit[0] and t >= unit[1]:           # a tile that slot 0 does not see: looked through before it is told of
                    self.v_at[st] = nk
                    self.v_full[st].arrive()
                else:
                    self.flying.append((self.v_full[st], st, nk))
                nk += 1
                yield

    def issue(self, s):
        nk = nq = np = 0
        for n, unit in enumerate(self.units + [None]):
            yield from self.wait(self.item_full[n & 1], n >> 1)
            if unit is None:
                return
            pair, cnt, other = unit[0], self.steps(unit, s), self.steps(unit, s ^ 1)
            if cnt + other > 0:
                yield from self.wait(self.q_full, nq)
                if cnt == 0:
                    self.q_empty.arrive()
                for u in range(-2, 2 * cnt):
                    i, h = u >> 1, u & 1
                    vt, kt = (nk + (2 * j + s if pair else j) for j in (i, i + 1))
                    if i >= 0:
                        waits = [(self.p_full[s][h], np)]
                        if h == 0:
                            waits.insert(1 if self.weights_first(u) else 0, (self.v_full[vt % self.NST], vt // self.NST))
                        for w in waits:
                            yield from self.wait(*w)
                        np += h
                        told = []
                        if h == 1:
                            told.append((self.v_empty[vt % self.NST], 2 if pair or i >= other else 1))
                            if i + 1 == cnt:
                                told.append((self.o_full[s], 1))
                        self.queue[s].append((vt, told))
                    if i + 1 < cnt and (h == 1 or not pair):
                        if h == 0 or pair:
                            yield from self.wait(self.k_full[kt % self.NST], kt // self.NST)
                        told = [(self.s_full[s][x], 1) for x in ((0, 1) if pair else (h,))]
                        if h == 1:
                            told.append((self.k_empty[kt % self.NST], 2 if pair or i + 1 >= other else 1))
                            if i + 2 == cnt:
                                told.append((self.q_empty, 1))
                        self.queue[s].append((None, told))
                nk += self.tiles(unit)
                nq += 1
            self.item_empty[n & 1].arrive()

    def softmax(self, s):
        ns = no = nj = 0
        unread = False
        for n, unit in enumerate(self.units + [None]):
            yield from self.wait(self.item_full[n & 1], n >> 1)
            if unit is None:
                return
            cnt = self.steps(unit, s)
            for i in range(cnt):
                if i == 0 and unread:
                    yield from self.wait(self.parted, nj - 1)
                    unread = False
                for h in range(2):
                    yield from self.wait(self.s_full[s][h], ns)
                    self.p_full[s][h].arrive()
                ns += 1
            if cnt > 0:
                yield from self.wait(self.o_full[s], no)
                no += 1
            if unit[0]:
                if self.join_waits and unread:
                    yield from self.wait(self.parted, nj - 1)
                    unread = False
                self.ml[s] = n
                self.joined.arrive()
                yield from self.wait(self.joined, nj)
                if self.ml[s ^ 1] != n:
                    raise Early("unit %d joined with the share of unit %s" % (n, self.ml[s ^ 1]))
                yield
                self.parted.arrive()
                nj += 1
                unread = True
            self.item_empty[n & 1].arrive()

    def land(self):
        barrier, st, tile = self.flying.pop(self.rng.randrange(len(self.flying)))
        if st is not None:
            self.v_at[st] = tile
        barrier.arrive()

    def compute(self, s):
        tile, told = self.queue[s].pop(0)
        if tile is not None and self.v_at[tile % self.NST] != tile:
            raise Early("tile %d of V used before it has landed" % tile)
        for barrier, n in told:
            barrier.arrive(n)

    def run(self):
        """One order of events, by chance: raises Early, or RuntimeError where nobody gets further."""
        actors = [self.copies(), self.issue(0), self.issue(1), self.softmax(0), self.softmax(1)]
        speed = [self.rng.random() ** 2 + 0.01 for _ in range(8)]     # of the actors, of copies, of the products of the two slots
        idle = 0
        while actors:
            can = list(range(len(actors))) + ([-1] if self.flying else []) + [-2 - s for s in (0, 1) if self.queue[s]]
            pick = self.rng.choices(can, [speed[c] for c in can])[0]
            if pick == -1:
                self.land()
            elif pick < -1:
                self.compute(-2 - pick)
            else:
                try:
                    next(actors[pick])
                except StopIteration:
                    actors.pop(pick)
                    speed.pop(pick)
            idle += 1
            if idle > 200000:
                raise RuntimeError("a wait that never ends")


def some_units(rng):
    """A few units: of few rows (tiles by turns), and of more rows, where slot 0 sees as many tiles as slot 1 or one less."""
    units = []
    for _ in range(rng.randrange(2, 6)):
        n = rng.randrange(0, 8)
        if rng.random() < 0.7:
            units.append((True, (n + 1) // 2, n // 2))
        else:
            units.append((False, max(n, 1) - rng.randrange(2), max(n, 1)))
    return units
