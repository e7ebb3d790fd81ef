"""A model of the waits of paged_tile_kernel on the CPU: producer, issuer, tensor pipe, memory and the two warpgroups over random items.

A wait on an mbarrier names a phase by its parity and passes where that one or any second one in front of it has ended, so a wait that is more than
a phase behind passes too early.  Here every wait also knows which phase it means: one that passes for another, a ring slot that is filled while it
is read or read before it is filled, scores or results that are overwritten before they are taken, and a circle of waits all fail."""
import os
import random
import re

import pytest

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2506_11498_b200", "csrc", "paged_attend.cu")


class Barrier:
    def __init__(self):
        self.ended = 0      # phases that have ended: the model's arrivals are one a phase

    def arrive(self):
        self.ended += 1

    def wait(self, parity, phase):
        """Passes as the hardware does; `phase`: the one that is meant."""
        while (self.ended & 1) == parity:
            yield
        assert self.ended == phase + 1, "a wait took phase %d for %d" % (self.ended - 1, phase)


class Model:
    def __init__(self, TQ, NS, items, seed, mistake=None):
        self.TQ, self.NS, self.items, self.rng, self.mistake = TQ, NS, items, random.Random(seed), mistake
        self.q_full, self.q_free = Barrier(), Barrier()
        self.kv_full, self.kv_empty = [Barrier() for _ in range(NS)], [Barrier() for _ in range(NS)]
        self.s_full, self.pv_done = [Barrier(), Barrier()], [Barrier(), Barrier()]
        self.p_full = [[Barrier(), Barrier()] for _ in "tt"]
        self.q = None                   # the item whose Q is there
        self.slot = [None] * NS         # the entry in each slot
        self.s = [None, None]           # what S holds: (item, tile, "scores" or the halves of P)
        self.o = [None, None]           # (item, tiles so far), "taken" when its warpgroup has read it
        self.loads, self.pipe = [], []
        self.votes = [0, 0]             # of the two warpgroups at their barrier

    # -- the order of tiles and entries --
    @staticmethod
    def tile_of(item, j):
        return item["t0"] + j if item["t0"] > 0 else (j + 1 if j + 1 < item["t1"] else 0)

    def entries(self, item, base, j):
        new = self.tile_of(item, j) == 0
        k = base + 2 * j
        return k, (k + 1 if new else None), k + (2 if new else 1)

    def after(self, item, base):
        return base + 2 * (item["t1"] - item["t0"]) + (1 if item["t0"] == 0 and self.mistake != "entries" else 0)

    # -- the roles --
    def producer(self):
        filled = 0
        for i, item in enumerate(self.items):
            if i > 0:
                yield from self.q_free.wait((i - 1) & 1, i - 1)
            self.loads.append(("q", i))
            n = item["t1"] - item["t0"] - (item["t0"] == 0)
            for _ in range(2 * n + (3 if item["t0"] == 0 else 0)):
                slot, use = filled % self.NS, filled // self.NS
                if filled >= self.NS and self.mistake != "full":
                    yield from self.kv_empty[slot].wait((use & 1) ^ 1, use - 1)
                self.loads.append((slot, filled))
                filled += 1
                yield

    def memory(self):
        while True:
            if self.loads:
                # (loads may land in any order)
                where, what = self.loads.pop(self.rng.randrange(len(self.loads)))
                if where == "q":
                    self.q = what
                    self.q_full.arrive()
                else:
                    assert self.slot[where] is None, "a slot is filled while it is read"
                    self.slot[where] = what
                    self.kv_full[where].arrive()
            yield

    def full(self, entry):
        return self.kv_full[entry % self.NS].wait(entry // self.NS & 1, entry // self.NS)

    def issuer(self):
        base, count = 0, [0, 0]
        for i, item in enumerate(self.items):
            n, tiles = item["t1"] - item["t0"], item["tiles"]
            yield from self.q_full.wait(i & 1, i)

            def wait_k(j):
                k, rest, _ = self.entries(item, base, j)
                yield from self.full(k)
                if rest is not None:
                    yield from self.full(rest)

            def scores(j, t):
                k, rest, _ = self.entries(item, base, j)
                self.pipe.append(("scores", t, i, j, [x for x in (k, rest) if x is not None]))
                self.pipe.append(("commit", self.s_full[t]))

            def free(entry):
                self.pipe.append(("free", entry))

            def free_k(j):
                k, rest, _ = self.entries(item, base, j)
                free(k)
                if rest is not None:
                    free(rest)
                if j + 1 == n:
                    self.pipe.append(("commit", self.q_free))

            def values(j, t, more):
                v = self.entries(item, base, j)[2]
                for half in range(2):
                    yield from self.p_full[t][half].wait(count[t] & 1, count[t])
                    self.pipe.append(("values", t, i, j, v, half, more))
                self.pipe.append(("commit", self.pv_done[t]))
                count[t] += 1

            if self.TQ == 2:
                for j in range(-1, n):
                    v = self.entries(item, base, j)[2] if j >= 0 else None
                    if j >= 0:
                        yield from self.full(v)
                    for t in range(tiles):
                        if j >= 0:
                            yield from values(j, t, j > 0)
                        if j + 1 < n:
                            if t == 0:
                                yield from wait_k(j + 1)
                            scores(j + 1, t)
                    if j >= 0:
                        free(v)
                    if j + 1 < n:
                        free_k(j + 1)
            else:
                for j in range(-2, n):
                    if j >= 0:
                        v = self.entries(item, base, j)[2]
                        yield from self.full(v)
                        yield from values(j, j & 1, j > 1)
                        free(v)
                    if j + 2 < n:
                        yield from wait_k(j + 2)
                        scores(j + 2, j & 1)
                        free_k(j + 2)
            base = self.after(item, base)

    def tensor(self):
        """The products and commits, in the order of issue."""
        while True:
            if self.pipe:
                op = self.pipe.pop(0)
                if op[0] == "scores":
                    _, t, i, j, entries = op
                    assert self.q == i and all(self.slot[e % self.NS] == e for e in entries), "operands that are not there"
                    assert self.s[t] is None, "scores over P that is still wanted"
                    self.s[t] = (i, j, "scores")
                elif op[0] == "values":
                    _, t, i, j, v, half, more = op
                    assert self.slot[v % self.NS] == v and self.s[t][:2] == (i, j) and half in self.s[t][2]
                    if half == 0:
                        assert more == (self.o[t] is not None and self.o[t] != "taken"), "results that were not taken"
                        self.o[t] = (i, (self.o[t][1] if more else 0) + 1)
                    else:
                        self.s[t] = None
                elif op[0] == "free":
                    entry = op[1]
                    assert self.slot[entry % self.NS] == entry
                    self.slot[entry % self.NS] = None
                    self.kv_empty[entry % self.NS].arrive()
                else:
                    op[1].arrive()
            yield

    def meet(self, t):
        self.votes[t] += 1
        while self.votes[t ^ 1] < self.votes[t]:
            yield

    def warpgroup(self, t):
        base, count, others = 0, 0, 0
        for i, item in enumerate(self.items):
            n = item["t1"] - item["t0"]
            mine = self.TQ == 1 or t < item["tiles"]
            first, step = (0, 1) if self.TQ == 2 else (t, 2)
            for j in range(first, n if mine else 0, step):
                v = self.entries(item, base, j)[2]
                yield from self.s_full[t].wait(count & 1, count)
                if self.tile_of(item, j) in item["ragged"]:      # rows of V to be zeroed
                    yield from self.full(v)
                    assert self.slot[v % self.NS] == v
                assert self.s[t] == (i, j, "scores")
                if j != first and self.rng.random() < 0.5:       # O is rescaled
                    yield from self.pv_done[t].wait((count - 1) & 1, count - 1)
                    assert self.o[t] == (i, (j - first) // step)
                for half in range(2):
                    self.s[t] = (i, j, (0,) if half == 0 else (0, 1))
                    self.p_full[t][half].arrive()
                    yield
                count += 1
            base = self.after(item, base)
            tiles = len(range(first, n, step))
            if mine and n > first:
                yield from self.pv_done[t].wait((count - 1) & 1, count - 1)
                assert self.o[t] == (i, tiles)
            if self.TQ == 1:
                theirs = n // 2 if t == 0 else (n + 1) // 2
                others += theirs
                if theirs > 0:
                    yield from self.pv_done[t ^ 1].wait((others - 1) & 1, others - 1)
                    assert self.o[t ^ 1] == (i, theirs)
                yield from self.meet(t)
                yield
                yield from self.meet(t)          # both have read both
                if n > first:
                    self.o[t] = "taken"
                yield from self.meet(t)
            elif mine:
                self.o[t] = "taken"

    def run(self):
        roles = [self.producer(), self.issuer(), self.warpgroup(0), self.warpgroup(1)]
        servants = [self.memory(), self.tensor()]
        idle = 0
        while roles:
            state = (len(self.loads), len(self.pipe), len(roles))
            before = self.progress()
            for agent in self.rng.sample(roles + servants, len(roles) + 2):
                for _ in range(self.rng.choice((1, 1, 4))):
                    try:
                        next(agent)
                    except StopIteration:
                        roles.remove(agent)
                        break
            idle = idle + 1 if self.progress() == before and state == (len(self.loads), len(self.pipe), len(roles)) else 0
            assert idle < 40, "a circle of waits"

    def progress(self):
        return (sum(b.ended for b in (self.q_full, self.q_free, *self.kv_full, *self.kv_empty, *self.s_full, *self.pv_done, *sum(self.p_full, []))),
                sum(self.votes), tuple(self.slot), tuple(map(str, self.s)))


def some_items(rng, TQ, most=9):
    """A CTA's runs: the first may begin inside an item, the last may end inside one."""
    items, n = [], rng.randint(1, 6)
    for i in range(n):
        tiles = rng.randint(1, most)
        t0 = rng.randint(0, tiles - 1) if i == 0 else 0
        t1 = rng.randint(t0 + 1, tiles) if i == n - 1 else tiles
        items.append(dict(t0=t0, t1=t1, tiles=rng.choice((1, 2)) if TQ == 2 else 1, ragged={0} | {t for t in range(1, tiles) if rng.random() < 0.3}))
    return items


FORMS = [(1, 8), (1, 5), (2, 8), (2, 3)]      # row tiles of a CTA, ring slots: d = 64 and 128


def test_the_forms_are_the_kernels():
    text = open(SOURCE).read()
    assert re.search(r"kStages = D == 64 \? 8 : TQ == 1 \? 5 : 3;", text)


@pytest.mark.parametrize("TQ, NS", FORMS)
def test_every_wait_means_the_phase_that_it_takes(TQ, NS):
    for seed in range(250):
        Model(TQ, NS, some_items(random.Random(seed), TQ), seed).run()


@pytest.mark.parametrize("TQ, NS", FORMS)
@pytest.mark.parametrize("mistake", ["entries", "full"])
def test_the_model_finds_mistakes(TQ, NS, mistake):
    """Entries of the new tokens' tile counted as a page's; a producer that does not wait for its slot."""
    found = 0
    for seed in range(40):
        try:
            Model(TQ, NS, some_items(random.Random(seed), TQ), seed, mistake).run()
        except AssertionError:
            found += 1
    assert found > 20
