"""The rings of the attention tiles over a pool held in 4 bits, as a model run under random schedules.

One actor copies raw parts, two make the stages of K and of V from them, one issues products, two are the softmax of either
row tile; segments are handed over through a ring of their own.  Where a row sees few keys a tile's keys take two stages of
K.  No schedule may leave an actor waiting, and every score and product is of the tile that it should be of."""
import random

import pytest


class Block:
    def __init__(self, seed, segments, k_stages, v_stages, parts, early=False):
        """segments: (tiles, two row tiles?, few keys?).  early: the issuer gives a tile's stages back before its products (a mistake)."""
        self.rng, self.segments = random.Random(seed), segments
        self.k_stages, self.v_stages, self.parts = k_stages, v_stages, parts
        self.early = early
        self.copied = self.k_took = self.v_took = 0            # raw parts
        self.k_free, self.v_free = k_stages, v_stages
        self.k_made, self.v_made = [], []                      # what the stages hold, in order: (segment, tile, rest?)
        self.k_used = self.v_used = 0
        self.handed = 0
        self.read = dict.fromkeys("copy k v issue soft0 soft1".split(), 0)
        self.scores, self.weights, self.products = set(), set(), set()
        self.errors = []

    def segment(self, who, i):
        yield lambda: self.handed > i
        self.read[who] = i + 1

    def hand_on(self):
        if self.handed < len(self.segments):
            yield lambda: min(self.read.values()) >= self.handed - 3       # a ring of four
            self.handed += 1

    def copy(self):
        yield from self.hand_on()
        for i, (n, _, _) in enumerate(self.segments):
            yield from self.segment("copy", i)
            yield from self.hand_on()
            for _ in range(4 * n):
                yield lambda: self.copied - min(self.k_took, self.v_took) < self.parts
                self.copied += 1

    def make_k(self):
        for i, (n, _, few) in enumerate(self.segments):
            yield from self.segment("k", i)
            for t in range(n):
                need = 2 if few else 1
                yield lambda: self.k_free >= need
                self.k_free -= need
                for _ in range(4):
                    yield lambda: self.copied > self.k_took
                    self.k_took += 1
                self.k_made += [(i, t, r) for r in range(2 if few else 1)]

    def make_v(self):
        for i, (n, _, _) in enumerate(self.segments):
            yield from self.segment("v", i)
            for t in range(n):
                yield lambda: self.v_free >= 1
                self.v_free -= 1
                for _ in range(4):
                    yield lambda: self.copied > self.v_took
                    self.v_took += 1
                self.v_made.append((i, t))

    def score(self, i, t, sub, stages):
        if [s for s in self.k_made[self.k_used: self.k_used + stages]] != [(i, t, r) for r in range(stages)]:
            self.errors.append("keys of another tile")
        self.scores.add((i, t, sub))

    def release(self, stages):
        self.k_used += stages
        self.k_free += stages

    def product(self, i, t, sub):
        yield lambda: (i, t, sub) in self.weights
        if self.v_made[self.v_used] != (i, t):
            self.errors.append("values of another tile")
        self.products.add((i, t, sub))

    def issue(self):
        for i, (n, two, few) in enumerate(self.segments):
            yield from self.segment("issue", i)
            subs, stages = range(2 if two else 1), 2 if few else 1
            ahead = 0 if few else 1 if two else 2
            made = 0
            for t in range(min(ahead, n)):
                yield lambda: len(self.k_made) >= self.k_used + 1
                for s in subs:
                    self.score(i, t, s, 1)
                self.release(1)
                made += 1
            for t in range(n):
                if few:
                    yield lambda: len(self.k_made) >= self.k_used + stages
                    if self.early:
                        self.release(stages)
                    for s in subs:
                        self.score(i, t, s, stages)
                    if not self.early:
                        self.release(stages)
                yield lambda: len(self.v_made) > self.v_used
                more = not few and made < n
                for s in subs:
                    yield from self.product(i, t, s)
                    if more:
                        if s == 0:
                            yield lambda: len(self.k_made) >= self.k_used + 1
                        self.score(i, made, s, 1)
                self.v_used += 1
                self.v_free += 1
                if more:
                    self.release(1)
                    made += 1

    def softmax(self, sub):
        for i, (n, two, _) in enumerate(self.segments):
            yield from self.segment("soft%d" % sub, i)
            if sub and not two:
                continue
            for t in range(n):
                yield lambda: (i, t, sub) in self.scores
                if t and self.rng.random() < 0.3:                          # the maximum moves: the products so far have to be there
                    yield lambda: (i, t - 1, sub) in self.products
                self.weights.add((i, t, sub))
            yield lambda: (i, n - 1, sub) in self.products

    def run(self):
        actors = {k: [f, None] for k, f in dict(copy=self.copy(), k=self.make_k(), v=self.make_v(), issue=self.issue(), s0=self.softmax(0), s1=self.softmax(1)).items()}
        while actors:
            ready = [k for k, (_, w) in actors.items() if w is None or w()]
            if not ready:
                return "stuck: " + " ".join(sorted(actors))
            k = self.rng.choice(ready)
            try:
                actors[k][1] = next(actors[k][0])
            except StopIteration:
                del actors[k]
        want = {(i, t, s) for i, (n, two, _) in enumerate(self.segments) for t in range(n) for s in range(2 if two else 1)}
        if self.products != want or self.k_free != self.k_stages or self.v_free != self.v_stages:
            self.errors.append("something is left")
        return " ".join(sorted(set(self.errors)))


def mixes(seed, rows):
    rng = random.Random(seed)
    return [(rng.randint(1, 6), rows == 256 and rng.random() < 0.7, rng.random() < 0.5) for _ in range(rng.randint(1, 9))]


@pytest.mark.parametrize("rows,k,v,parts", [(256, 2, 2, 5), (128, 2, 2, 12), (256, 4, 4, 5), (128, 4, 4, 12)])
def test_every_schedule_ends(rows, k, v, parts):
    for seed in range(120):
        assert Block(seed, mixes(seed, rows), k, v, parts).run() == "", (seed, mixes(seed, rows))


def test_the_model_sees_mistakes():
    # with a single stage of K, two for one tile never come
    assert Block(1, [(1, True, True)], 1, 2, 5).run().startswith("stuck")
    # stages that are given back before their products are read hold another tile by then
    assert any(Block(s, [(3, True, True)], 2, 2, 5, early=True).run() for s in range(50))
    # a ring of raw parts that holds less than a tile needs both makers at its pace, and has them
    assert Block(2, [(4, False, True)], 2, 2, 1).run() == ""
