"""The page pool's copies taken together: pairs of several extends in one call, and a step that runs out of pages."""
import os
import random
import sys

import pytest

A = pytest.importorskip("paper_2606_12876_amd", reason="libaqmb.so not built")

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
from decode_step import Streams  # noqa: E402


class Memory:
    """What a cache holds, by slot, and what every sequence wrote."""

    def __init__(self, n_pages, size):
        self.size, self.pages, self.text, self.stamp = size, [[None] * size for _ in range(n_pages)], {}, 0

    def copy(self, pairs):
        """All at once, as the kernel does: pages that are read must not be written."""
        src, dst = [p[0] for p in pairs], [p[1] for p in pairs]
        assert len(set(dst)) == len(dst) and not set(src) & set(dst), pairs
        for (_, d), page in zip(pairs, [list(self.pages[s]) for s in src]):
            self.pages[d] = page

    def write(self, seq, slots):
        for slot in slots:
            self.stamp += 1
            self.pages[slot // self.size][slot % self.size] = self.stamp
            self.text[seq].append(self.stamp)

    def check(self, pool):
        for seq, text in self.text.items():
            table = pool.table(seq).tolist()
            assert pool.length(seq) == len(text)
            assert [self.pages[table[t // self.size]][t % self.size] for t in range(len(text))] == text


@pytest.mark.parametrize("seed", range(8))
def test_copies_of_extends_in_a_row(seed):
    """Every stream extended, the pairs copied in one call, the tokens written; forks and frees between the steps."""
    rng = random.Random(seed)
    n_pages, size = rng.choice([(30, 4), (60, 7), (90, 16)])
    pool, mem = A.PagePool(n_pages, size, 12), Memory(n_pages, size)
    for _ in range(200):
        if rng.random() < 0.3 and len(mem.text) < 12:
            old = rng.choice([None] + sorted(mem.text))
            new = pool.add() if old is None else pool.fork(old)
            mem.text[new] = [] if old is None else list(mem.text[old])
        pairs, todo = [], []
        for s in sorted(mem.text, key=lambda _: rng.random()):
            try:
                slots, copies = pool.extend(s, rng.choice([0, 1, 1, size, 2 * size + 1]))
            except A.AqmbError:
                continue
            pairs += copies
            todo.append((s, slots.tolist()))
        mem.copy(pairs)
        for s, slots in todo:
            mem.write(s, slots)
        mem.check(pool)
        while mem.text and pool.counts()[0] < rng.randint(0, 9):
            s = rng.choice(sorted(mem.text))
            pool.free(s)
            del mem.text[s]
            mem.check(pool)


class OnTheHost(Streams):
    def __init__(self, pool, mem):
        super().__init__(pool, [], device="cpu")
        self.mem = mem

    def copy(self, pairs):
        self.mem.copy(pairs)


def step(streams, mem, seqs):
    positions, slots, table, lengths, most = streams.advance(seqs)
    for i, s in enumerate(seqs):
        assert positions[i] == len(mem.text[s]) and lengths[i] == len(mem.text[s]) + 1 <= most
        mem.write(s, [int(slots[i])])
    mem.check(streams.pool)


def test_a_step_without_enough_pages():
    """Streams 0 and 1 share a page, so do 2 and 3, 4 has one; copies for 0 and 2 need two pages and one is free."""
    pool, mem = A.PagePool(4, 4, 5), Memory(4, 4)
    streams = OnTheHost(pool, mem)

    def add():
        new = pool.add()
        mem.text[new] = []
        return new

    def free(s):
        streams.free(s)
        del mem.text[s]

    def runs_out(seqs):
        with pytest.raises(A.AqmbError) as e:
            streams.advance(seqs)
        assert e.value.status == A.Status.ENOMEM

    for _ in range(2):
        new = add()
        step(streams, mem, [new])
        step(streams, mem, [new])
        mem.text[pool.fork(new)] = list(mem.text[new])
    step(streams, mem, [add()])
    assert sorted(mem.text) == [0, 1, 2, 3, 4]
    runs_out([0, 2, 3])
    free(1)                                 # gives the page back that 0 copies from
    step(streams, mem, [0, 2, 3])
    step(streams, mem, [0, 2, 3])           # three full pages now
    free(4)
    runs_out([2, 0, 3])
    free(2)                                 # extended in the step that failed
    assert add() == 1 and add() == 2
    step(streams, mem, [2, 3])
    runs_out([0])
    free(3)
    step(streams, mem, [0, 2, 1])
    assert not streams.ready
