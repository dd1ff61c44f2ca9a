"""The bookkeeping of a cache's pages, against a model that keeps every sequence's tokens as a list and the cache as an array of them (no GPU needed)."""
import random

import pytest

from paper_2205_14135_amd.paged import OutOfPages, PageTable


class Model:
    def __init__(self, pages, page_size):
        self.table, self.size = PageTable(pages, page_size), page_size
        self.cache = [[None] * page_size for _ in range(pages)]
        self.tokens = {}

    def copy(self, pairs):
        src, dst = {s for s, _ in pairs}, [d for _, d in pairs]
        assert len(set(dst)) == len(dst) and not src & set(dst)          # what attn_paged_copy asks for
        for s, d in pairs:
            self.cache[d] = list(self.cache[s])

    def extend(self, seqs, new):
        self.copy(self.table.extend(seqs, [len(n) for n in new]))
        for s, n in zip(seqs, new):
            for t in n:
                at = len(self.tokens[s])
                self.cache[self.table.pages_of(s)[at // self.size]][at % self.size] = t
                self.tokens[s].append(t)

    def check(self):
        used = set()
        for s, want in self.tokens.items():
            held = self.table.pages_of(s)
            assert self.table.length(s) == len(want) and len(held) == -(-len(want) // self.size) and len(set(held)) == len(held)
            assert [self.cache[held[i // self.size]][i % self.size] for i in range(len(want))] == want
            used |= set(held)
        assert self.table.free_pages == self.table.pages - len(used)
        return used


@pytest.mark.parametrize("seed", range(12))
def test_random_programs(seed):
    rng = random.Random(seed)
    m = Model(rng.choice([5, 12, 40]), 16)
    count = 0
    for _ in range(300):
        what = rng.random()
        live = list(m.tokens)
        if what < 0.2 or not live:
            m.tokens[m.table.add()] = []
        elif what < 0.35:
            s = rng.choice(live)
            m.tokens[m.table.fork(s)] = list(m.tokens[s])
        elif what < 0.5:
            s = rng.choice(live)
            m.table.free(s)
            del m.tokens[s]
        elif what < 0.6:
            pairs = m.table.compact()
            m.copy(pairs)
            used = m.check()
            assert used == set(range(len(used)))
        else:
            seqs = rng.sample(live, rng.randint(1, len(live)))
            new = []
            for _ in seqs:
                n = rng.choice([0, 1, 1, 3, 16, 40])
                new.append(list(range(count, count + n)))
                count += n
            before = (m.table.free_pages, {s: m.table.pages_of(s) for s in live})
            try:
                m.extend(seqs, new)
            except OutOfPages:
                assert before == (m.table.free_pages, {s: m.table.pages_of(s) for s in live})
        m.check()


def test_the_last_writer_of_a_shared_page_keeps_it():
    t = PageTable(8, 16)
    a = t.add()
    assert t.extend([a], [20]) == []
    b = t.fork(a)
    assert t.extend([a, b], [1, 1]) == [(1, 2)] and t.pages_of(a) == [0, 2] and t.pages_of(b) == [0, 1]
    c = t.fork(a)
    assert t.extend([c], [0]) == [] and t.extend([a], [11]) == [(2, 3)]           # nothing written, nothing copied
    assert t.extend([c], [12]) == [] and t.pages_of(c) == [0, 2, 4]
    t.free(a), t.free(b), t.free(c)
    assert t.free_pages == 8


def test_full_pages_are_shared_without_copies():
    t = PageTable(4, 16)
    a = t.add()
    t.extend([a], [32])
    b = t.fork(a)
    assert t.extend([a, b], [1, 1]) == [] and t.pages_of(a) == [0, 1, 2] and t.pages_of(b) == [0, 1, 3]


def test_batch():
    t = PageTable(6, 32)
    a, b, c = t.add(), t.add(), t.add()
    t.extend([a, b], [40, 7])
    table, lengths = t.batch([b, a, c], device="cpu")
    assert table.tolist() == [[2, -1], [0, 1], [-1, -1]] and lengths.tolist() == [7, 40, 0]
    assert str(table.dtype) == str(lengths.dtype) == "torch.int32"
    table, lengths = t.batch([], device="cpu")
    assert table.shape == (0, 1) and lengths.shape == (0,)


def test_refusals():
    for pages, size in ((0, 16), (4, 8), (4, 24), (4, 8192)):
        with pytest.raises(ValueError):
            PageTable(pages, size)
    t = PageTable(2, 16)
    a = t.add()
    for seqs, tokens in (([a], [1, 2]), ([a, a], [1, 1]), ([a], [-1])):
        with pytest.raises(ValueError):
            t.extend(seqs, tokens)
    with pytest.raises(OutOfPages):
        t.extend([a], [33])
    assert t.free_pages == 2 and t.length(a) == 0
    with pytest.raises(KeyError):
        t.extend([7], [1])
    t.free(a)
    with pytest.raises(KeyError):
        t.free(a)
