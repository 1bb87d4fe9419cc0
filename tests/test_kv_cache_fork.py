"""FqKvCache's shared pages: forking, copying before writing, compacting and freeing, with the calls replaced by plain copies (no GPU needed)."""
import random

import pytest
import torch

import paper_2402_17985_amd as fq
from paper_2402_17985_amd import binding


@pytest.fixture
def copies(monkeypatch):
    """fq_kv_copy_pages in torch, with its contract checked; fq_kv_append writes each token's number into its slot of k_cache."""
    seen = []

    def copy(k, v, ks, vs, src, dst, stream=None):
        src, dst = src.tolist(), dst.tolist()
        assert len(set(dst)) == len(dst) and not set(src) & set(dst) and all(0 <= p < len(k) for p in src + dst)
        for t in (k, v, ks, vs):
            t[dst] = t[src].clone()
        seen.append((src, dst))

    def append(Q, K, V, cu, past, most, k_cache, v_cache, ks, vs, table, **_):
        page, cu, past = k_cache.shape[2], cu.tolist(), past.tolist()
        written = set()
        for b, n in enumerate(past):
            for i in range(cu[b + 1] - cu[b]):
                at = n + i
                p = int(table[b, at // page])
                written.add((b, p))
                k_cache[p, 0, at % page] = K[cu[b] + i, 0]
        pages = [p for _, p in written]
        assert len(set(pages)) == len(pages)      # no two sequences write into one page

    monkeypatch.setattr(binding, "fq_kv_copy_pages", copy)
    monkeypatch.setattr(binding, "fq_kv_append", append)
    return seen


class Model:
    """What each sequence should hold, beside the cache."""

    def __init__(self, pages, batch, max_len=512):
        self.cache, self.tokens, self.next = fq.FqKvCache(pages, batch, max_len, 1, 64, device="cpu"), [[] for _ in range(batch)], 0
        self.cache.k_cache.zero_()

    def append(self, new):
        fresh = [[(self.next + sum(new[:b]) + i) % 127 for i in range(n)] for b, n in enumerate(new)]
        rows = torch.tensor([t for f in fresh for t in f], dtype=torch.int8)[:, None, None].expand(-1, 1, 64)
        self.cache.append(None, rows, rows, new)
        self.next += sum(new)
        for t, f in zip(self.tokens, fresh):
            t += f

    def fork(self, b, into):
        self.cache.fork(b, into)
        for c in into:
            self.tokens[c] = list(self.tokens[b])

    def release(self, b):
        self.cache.release(b)
        self.tokens[b] = []

    def drop(self, b, n):
        self.tokens[b] = self.tokens[b][:n]
        self.cache.lengths[b] = n

    def check(self):
        c = self.cache
        users = [0] * len(c.k_cache)
        for b, want in enumerate(self.tokens):
            assert c.lengths[b] == len(want) and len(c.held[b]) >= -(-len(want) // 64)
            assert c.page_table[b].tolist() == c.held[b] + [-1] * (c.page_table.shape[1] - len(c.held[b]))
            assert [int(c.k_cache[c.held[b][i // 64], 0, i % 64, 0]) for i in range(len(want))] == want
            for p in c.held[b]:
                users[p] += 1
        assert users == c._users and sorted(c._free) == [p for p, n in enumerate(users) if n == 0]


def test_forks_share_and_copy_what_they_change(copies):
    m = Model(12, 4)
    m.append([100, 0, 0, 0])
    m.fork(0, [1, 2])
    m.check()
    assert len(m.cache._free) == 10 and not copies      # two pages, held three times
    m.append([1, 1, 0, 0])                              # two of the three go on: both take copies of the page that is partly filled
    m.check()
    assert copies == [([m.cache.held[2][1]] * 2, [m.cache.held[0][1], m.cache.held[1][1]])]
    m.append([0, 0, 1, 0])                              # the third has it for itself now
    m.check()
    assert len(copies) == 1
    m.release(0)
    m.release(2)
    m.check()
    assert [int(n) for n in m.cache._users].count(1) == 2


def test_all_holders_go_on(copies):
    """The last one keeps the page: with two holders one copy is made, and one page is taken."""
    m = Model(4, 2)
    m.append([70, 0])
    m.fork(0, [1])
    m.append([2, 3])
    m.check()
    assert len(copies) == 1 and len(copies[0][0]) == 1 and len(m.cache._free) == 1


def test_a_page_begun_anew_is_not_copied(copies):
    """After rejected drafts a sequence may write into shared pages behind its own last token."""
    m = Model(12, 2)
    m.append([200, 0])
    m.fork(0, [1])
    m.drop(1, 64)
    m.append([0, 100])
    m.check()
    assert not copies
    m.drop(0, 130)
    m.append([1, 0])
    m.check()


def test_a_full_page_is_never_copied(copies):
    m = Model(6, 2)
    m.append([128, 0])
    m.fork(0, [1])
    m.append([5, 5])
    m.check()
    assert not copies and m.cache.held[0][:2] == m.cache.held[1][:2]


def test_too_few_pages_change_nothing(copies):
    m = Model(3, 3)
    m.append([70, 0, 0])
    m.fork(0, [1, 2])
    before = (list(m.cache._free), [list(h) for h in m.cache.held], list(m.cache._users))
    with pytest.raises(RuntimeError, match="2 pages wanted, 1 free"):
        m.append([1, 1, 1])
    assert before == (m.cache._free, m.cache.held, m.cache._users)
    m.append([1, 0, 0])
    m.check()


def test_pages_reserved_ahead_stay_with_their_sequence(copies):
    m = Model(8, 2)
    m.cache.reserve(0, 300)
    m.append([10, 0])
    m.fork(0, [1])
    assert len(m.cache.held[0]) == 5 and len(m.cache.held[1]) == 1
    m.append([100, 0])
    m.append([0, 60])
    m.check()


def test_nothing_to_fork(copies):
    m = Model(4, 3)
    m.fork(0, [1, 2])
    m.fork(1, [])
    m.check()
    with pytest.raises(ValueError):
        m.cache.fork(0, [1, 1])
    for b, into in ((0, [3]), (0, [-1]), (5, [0])):
        with pytest.raises(ValueError):
            m.cache.fork(b, into)
    m.append([1, 1, 0])
    with pytest.raises(ValueError, match="release"):
        m.cache.fork(0, [1])
    with pytest.raises(ValueError, match="release"):
        m.cache.fork(0, [0])


def test_compact(copies):
    m = Model(20, 4)
    m.append([130, 70, 200, 10])
    m.fork(2, [])
    m.release(1)
    m.release(0)
    assert m.cache.compact() == 5
    m.check()
    assert sorted(set(sum(m.cache.held, []))) == [0, 1, 2, 3, 4] and m.cache._free[-1] == 5
    assert m.cache.compact() == 5 and len(copies) == 1              # nothing left to move
    m.fork(2, [0])
    m.release(2)
    m.append([30, 0, 0, 0])
    m.check()
    assert fq.FqKvCache(4, 1, 64, 1, 64, device="cpu").compact() == 0


@pytest.mark.parametrize("seed", range(20))
def test_any_order_of_calls(copies, seed):
    r = random.Random(seed)
    m = Model(40, 5, max_len=640)
    for _ in range(60):
        kind = r.choice(["append", "append", "append", "fork", "release", "drop", "compact"])
        b = r.randrange(5)
        if kind == "append":
            try:
                m.append([r.choice([0, 0, 1, 5, 64, 90]) for _ in range(5)])
            except RuntimeError:
                m.release(b)
        elif kind == "fork":
            m.fork(b, [c for c in range(5) if not m.cache.held[c] and c != b][: r.randrange(3)])
        elif kind == "release":
            m.release(b)
        elif kind == "drop" and m.tokens[b]:
            m.drop(b, r.randrange(len(m.tokens[b]) + 1))
        elif kind == "compact":
            m.cache.compact()
        m.check()
