"""The barriers between the roles of a walk on the tensor cores: a wait looks at one bit of a barrier's phase, so that a role which is two phases
behind waits for one that never comes.  The roles' waits and arrivals in the order of the kernel, run side by side on the host in many
orders: no wait may find its barrier two phases on, and all of them end.  How many barriers there are of a kind is read from the source."""
import os
import random
import re

import pytest

import paper_1911_00472_b200

TILE = 128


def _barriers():
    with open(os.path.join(os.path.dirname(paper_1911_00472_b200.__file__), "csrc", "pcr_decay_tiles.cuh")) as f:
        names = re.search(r"uint64_t (full[^;]+);", f.read()).group(1)
    return {m[0]: int(m[1] or 1) for m in re.findall(r"(\w+)(?:\[(\d+)\])?(?:, |$)", names)}


class Walk:
    """One CTA over segments of `jobs` tokens; roles are generators, what they yield has to be true before they go on."""

    def __init__(self, jobs, given, places, per, rng):
        self.jobs, self.given, self.places, self.per, self.rng = jobs, given, places, per, rng
        self.kinds = _barriers()
        self.phase, self.arrived, self.posted = {}, {}, 0

    def arrive(self, name, i=0, count=1):
        self.arrived[name, i] = self.arrived.get((name, i), 0) + 1
        if self.arrived[name, i] == count:
            self.arrived[name, i] = 0
            self.phase[name, i] = self.phase.get((name, i), 0) + 1

    def wait(self, name, i, n):
        """For the n-th phase (from 0) of a barrier to end."""
        def there():
            done = self.phase.get((name, i), 0)
            assert done <= n + 1, f"{name}[{i}]: phase {n} is waited for when {done} have ended"
            return done == n + 1
        return there

    def chunks(self):
        """(chunk over all segments, tokens, whether it is added to the memory)"""
        g = 0
        for j, n in enumerate(self.jobs):
            c = -(-n // TILE)
            for i in range(c):
                yield j, i, g, min(TILE, n - TILE * i), i < (c if self.given[j] else c - 1)
                g += 1

    def of_job(self, j):
        return [x for x in self.chunks() if x[0] == j]

    def next(self, j):
        """Give the segment before back, wait for this one."""
        if j > 0:
            self.arrive("taken", (j - 1) % 3, 5)                     # (five roles here; a role's warps go on together in this model)
        return self.wait("got", j % 3, j // 3)

    def segments(self):
        for j in range(len(self.jobs) + 1):
            if j >= 3:
                yield self.wait("taken", j % 3, j // 3 - 1)
            self.arrive("got", j % 3)

    def copies(self):
        for j in range(len(self.jobs) + 1):
            yield self.next(j)
            for _, _, g, _, _ in self.of_job(j):
                for which in range(self.per):
                    at = g * self.per + which
                    if at >= self.places:
                        yield self.wait("empty", at % self.places, at // self.places - 1)
                    self.arrive("full", at % self.places)

    def tile(self, g, which):
        at = g * self.per + which
        return self.wait("full", at % self.places, at // self.places)

    def free(self, g, which):
        self.arrive("empty", (g * self.per + which) % self.places)

    def products(self):
        todo = list(self.chunks())
        b, c = (1, 2) if self.per == 3 else (0, 1)
        slots, tails, known, ahead = self.kinds["z"], 0, 0, False

        def know(j):                                                  # (segments without a chunk are none of this model's)
            return self.next(j)

        for x, (j, i, g, n, adds) in enumerate(todo):
            if i == 0 and known == j:
                yield know(j)
                known = j + 1
            if not ahead:
                yield self.tile(g, 0)
                yield self.tile(g, b)
                if g:
                    yield self.wait("o", 0, g - 1)
                self.arrive("s", g & 1)
            ahead = False
            yield self.tile(g, c)
            if n < TILE:
                yield self.wait("z", tails % slots, tails // slots)
                tails += 1
            yield self.wait("p", 0, g)
            if g:
                yield self.wait("e", 0, g - 1)
            self.arrive("o", 0)
            if x + 1 < len(todo) and self.rng.random() < 0.7:         # the next S, where its segment and tiles are there already
                nj, ni, ng, _, _ = todo[x + 1]
                if ni == 0 and known == nj and self.phase.get(("got", nj % 3), 0) > nj // 3:
                    yield know(nj)
                    known = nj + 1
                if known > nj and self.tile(ng, 0)() and self.tile(ng, b)():
                    yield self.wait("o", 0, g)
                    self.arrive("s", ng & 1)
                    ahead = True
            yield self.wait("r", 0, g)
            self.arrive("i", g & 1)
            if b:
                self.free(g, 0)
            yield self.wait("k", 0, g)
            self.arrive("d", 0)
            self.free(g, b)
            self.free(g, c)
        yield know(len(self.jobs))

    def parts(self):
        b, c = (1, 2) if self.per == 3 else (0, 1)
        slots, tails = self.kinds["z"], 0
        for j in range(len(self.jobs) + 1):
            yield self.next(j)
            for _, _, g, n, adds in self.of_job(j):
                yield self.tile(g, b)
                if n < TILE:
                    yield self.tile(g, c)
                    self.arrive("z", tails % slots)
                    tails += 1
                if g:
                    yield self.wait("d", 0, g - 1)
                yield self.wait("s", g & 1, g >> 1)
                if self.given[j]:
                    yield self.wait("i", g & 1, g >> 1)
                self.arrive("k", 0)

    def memory(self):
        for j in range(len(self.jobs) + 1):
            yield self.next(j)
            todo = self.of_job(j)
            for x in range(len(todo) + 1):
                if x:
                    yield self.wait("d", 0, todo[x - 1][2])
                if x < len(todo):
                    self.arrive("r", 0)

    def rows(self):
        for j in range(len(self.jobs) + 1):
            yield self.next(j)
            todo = self.of_job(j)
            for x in range(len(todo)):
                for y in ([x] if x == 0 else []) + ([x + 1] if x + 1 < len(todo) else []):
                    yield self.wait("s", todo[y][2] & 1, todo[y][2] >> 1)
                    self.arrive("p", 0)
                yield self.wait("i", todo[x][2] & 1, todo[x][2] >> 1)
                self.arrive("e", 0)

    def run(self):
        roles = [r() for r in (self.segments, self.copies, self.products, self.parts, self.memory, self.rows)]
        pace = [self.rng.choice([0.02, 0.2, 1.0, 1.0]) for _ in roles]   # some much slower than others
        waits = [None] * len(roles)
        left = set(range(len(roles)))
        idle = 0
        while left:
            i = self.rng.choice(sorted(left))
            if self.rng.random() > pace[i]:
                continue
            if waits[i] is not None and not waits[i]():
                idle += 1
                assert idle < 100000, "nothing goes on"
                continue
            idle = 0
            try:
                waits[i] = next(roles[i])
            except StopIteration:
                left.discard(i)


@pytest.mark.parametrize("places,per", [(5, 3), (6, 2)])
@pytest.mark.parametrize("kind", ["short", "mixed", "long"])
def test_no_role_falls_two_phases_behind(kind, places, per):
    rng = random.Random(places + len(kind))
    lengths = {"short": [1, 5, 61, 127], "mixed": [1, 127, 128, 129, 255, 256, 300], "long": [700, 128, 1000, 513]}[kind]
    for _ in range(150):
        jobs = [rng.choice(lengths) for _ in range(rng.randint(1, 9))]
        Walk(jobs, [rng.random() < 0.4 for _ in jobs], places, per, rng).run()
