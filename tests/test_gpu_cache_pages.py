"""si_cache_trim / _extend / _fork / _compact against the same calls on Python integers: tables, lengths, reference counts and the content of
every page (free ones too: nothing else may be written) are equal after each call."""
import random

import numpy as np
import pytest
import torch

import paper_2411_15715_amd as si
from attention_reference import Books, Cache

pytestmark = pytest.mark.gpu
BF, F8 = si.SI_KV_BF16, si.SI_KV_E4M3


def dev(a):
    return torch.tensor(list(a), dtype=torch.int32, device="cuda")


class Pool:
    def __init__(self, kind=BF, n_pages=40, page=32, n_seqs=8, max_pages=12, n_layers=2, kv_heads=1, d=64, seed=0):
        if kind == F8:
            page = max(page, 64)
        self.c = Cache(kind, n_pages, page, n_seqs, max_pages, n_layers, kv_heads, d, None, seed)
        self.original = self.c.bits().reshape(n_pages, -1).copy()
        self.scratch = torch.zeros(si.si_cache_scratch_bytes(self.c.desc), dtype=torch.uint8, device="cuda")
        self.c.desc.scratch = self.scratch.data_ptr()
        self.books = Books(self.c)
        self.stream = torch.cuda.current_stream().cuda_stream

    def check(self, status=0):
        torch.cuda.synchronize()
        b, c = self.books, self.c
        assert int(c.status.item()) == status
        c.status.zero_()
        assert np.array_equal(c.lens.cpu().numpy(), b.lens)
        assert np.array_equal(c.table.cpu().numpy(), b.table)
        assert np.array_equal(c.refs.cpu().numpy(), b.refs)
        bits = c.bits().reshape(len(b.refs), -1)
        wrong = [p for p in range(len(b.refs)) if not np.array_equal(bits[p], self.original[b.content[p]])]
        assert not wrong, "pages with another content: %s" % wrong

    def trim(self, seqs, keep=None):
        status = self.books.trim(seqs, keep)
        s, k = dev(seqs), dev(keep) if keep is not None else None
        si.si_cache_trim(self.c.desc, s.data_ptr(), len(seqs), k.data_ptr() if k is not None else None, self.stream)
        self.check(status)

    def extend(self, seqs, counts, capacity=None, uniform=False):
        capacity = sum(max(c, 0) for c in counts) if capacity is None else capacity
        want, status = self.books.extend(seqs, counts, capacity)
        s, k = dev(seqs), dev(counts)
        seq, pos = (torch.full((capacity + 2,), 7, dtype=torch.int32, device="cuda") for _ in range(2))
        si.si_cache_extend(self.c.desc, s.data_ptr(), len(seqs), None if uniform else k.data_ptr(), counts[0] if uniform else 0, seq.data_ptr(), pos.data_ptr(),
                           capacity, self.stream)
        self.check(status)
        assert list(zip(seq.tolist(), pos.tolist())) == want + [(7, 7)] * 2
        return status

    def fork(self, parents, children):
        status = self.books.fork(parents, children)
        a, b = dev(parents), dev(children)
        si.si_cache_fork(self.c.desc, a.data_ptr(), b.data_ptr(), len(parents), self.stream)
        self.check(status)
        return status

    def compact_in_place(self):
        place, m = self.books.compact()
        used = torch.full((1,), -1, dtype=torch.int32, device="cuda")
        si.si_cache_compact(self.c.desc, self.c.desc, used.data_ptr(), self.stream)
        b = self.books
        refs, content = np.zeros_like(b.refs), b.content.copy()
        for p in np.flatnonzero(place >= 0):
            refs[place[p]], content[place[p]] = b.refs[p], b.content[p]
        b.table, b.refs, b.content = np.where(b.table >= 0, place[np.maximum(b.table, 0)], -1), refs, content
        self.check()
        assert int(used.item()) == m


@pytest.mark.parametrize("kind", [BF, F8])
def test_grow_trim_and_free(kind):
    p = Pool(kind)
    page = p.c.page
    p.extend([0, 3, 5], [5, page, 2 * page + 1])
    p.extend([5, 0], [1, page - 5])
    p.extend([0], [1])
    p.trim([5, 3], [page, page - 1])
    p.extend([3, 1, 5], [1, 3 * page, 0])
    p.trim([0, 1])
    p.trim([3, 5], [0, 1])
    p.extend([7, 6, 5, 4], [4, 4, 4, 4], uniform=True)


def test_pages_are_taken_in_ascending_order():
    p = Pool()
    p.extend([0, 1, 2], [32 * 3] * 3)
    p.trim([1])
    p.extend([5], [32 * 4])
    assert p.c.table[5, :4].tolist() == [3, 4, 5, 9]


def test_forks_share_full_pages_and_copy_the_last():
    p = Pool()
    p.extend([0, 1], [32 * 2 + 7, 32 * 2])
    p.fork([0, 1, 0, 0], [2, 3, 4, 5])
    p.extend([2, 0, 3, 1], [40, 1, 1, 33])
    p.trim([0])
    p.trim([2, 4], [3, 64])
    p.fork([5], [0])


def test_a_shared_partial_page_is_copied_before_it_grows():
    """Trimmed into a page that others share: every sharer but the last gets a copy, wherever in the list it is."""
    p = Pool(n_pages=60)
    p.extend([0], [32 * 3])
    p.fork([0, 0, 0, 0], [1, 2, 3, 4])
    p.trim([0, 1, 2, 3], [70, 71, 65, 95])
    p.extend([2, 0], [1, 1])
    p.extend([3, 1, 4], [1, 60, 1])
    p.trim([4, 3, 2], [1, 1, 1])
    p.extend([4, 3, 2, 0], [0, 31, 1, 1])
    p.trim([0, 1, 2, 3, 4])


def test_errors_leave_everything_as_it_was():
    p = Pool(n_pages=6)
    p.extend([0, 1], [40, 20])
    assert p.extend([2], [32 * 4]) == si.SI_CACHE_NO_PAGES
    assert p.extend([2, 0], [1, 32 * 3]) == si.SI_CACHE_NO_PAGES
    assert p.extend([2, 8], [1, 1]) == si.SI_CACHE_BAD_SEQ
    assert p.extend([-1], [1]) == si.SI_CACHE_BAD_SEQ
    assert p.extend([2, 3, 2], [1, 1, 1]) == si.SI_CACHE_BAD_SEQ
    assert p.extend([2, 1], [1, -1]) == si.SI_CACHE_BAD_LEN
    assert p.extend([1], [32 * 12 - 19]) == si.SI_CACHE_BAD_LEN
    assert p.extend([1], [0x7fffffff], capacity=4) == si.SI_CACHE_BAD_LEN
    assert p.extend([1, 2], [4, 4], capacity=7) == si.SI_CACHE_NO_ROOM
    assert p.extend([1, 2], [4, 4], capacity=11) == 0
    p.trim([1, 9, -3], [25, 0, 0])
    p.trim([1, 0], [-1, 3])
    assert p.fork([0, 1], [3, 3]) == si.SI_CACHE_BAD_SEQ
    assert p.fork([0, 3], [3, 4]) == si.SI_CACHE_BAD_SEQ
    assert p.fork([0], [0]) == si.SI_CACHE_BAD_SEQ
    assert p.fork([0], [8]) == si.SI_CACHE_BAD_SEQ
    assert p.fork([-1], [3]) == si.SI_CACHE_BAD_SEQ
    assert p.fork([0], [1]) == si.SI_CACHE_BAD_LEN
    assert p.fork([0, 0, 0, 1], [3, 4, 5, 6]) == si.SI_CACHE_NO_PAGES
    assert p.fork([0, 0, 1], [3, 4, 6]) == 0


def test_spoilt_tables_and_counts():
    """Page numbers and counts that cannot be: never followed."""
    p = Pool()
    p.extend([0, 1], [100, 40])
    for entry in (-1, 40, 0x7fffffff, -0x80000000):
        keep = int(p.c.table[0, 1])
        p.c.table[0, 1] = entry
        before = p.c.bits().copy()
        a, b = dev([0]), dev([3])
        si.si_cache_fork(p.c.desc, a.data_ptr(), b.data_ptr(), 1, p.stream)
        torch.cuda.synchronize()
        assert int(p.c.status.item()) == si.SI_CACHE_BAD_PAGE and np.array_equal(p.c.bits(), before)
        p.c.status.zero_()
        p.c.table[0, 1] = keep
        p.check()
        keep = int(p.c.table[1, 1])
        p.c.table[1, 1] = entry
        a = dev([1])
        si.si_cache_extend(p.c.desc, a.data_ptr(), 1, None, 1, None, None, 0, p.stream)
        torch.cuda.synchronize()
        assert int(p.c.status.item()) == si.SI_CACHE_BAD_PAGE
        p.c.status.zero_()
        p.c.table[1, 1] = keep
        p.check()
    for length in (-1, -0x80000000, 32 * 12 + 1, 0x7fffffff):
        p.c.lens[1] = length
        a, b = dev([1]), dev([3])
        si.si_cache_extend(p.c.desc, a.data_ptr(), 1, None, 1, None, None, 0, p.stream)
        si.si_cache_fork(p.c.desc, a.data_ptr(), b.data_ptr(), 1, p.stream)
        torch.cuda.synchronize()
        assert int(p.c.status.item()) == si.SI_CACHE_BAD_LEN
        p.c.status.zero_()
        p.c.lens[1] = 40
        p.check()
    # a page in use with no count: trimming reports it and the count stays at 0; an entry outside the pool is dropped
    p.c.refs[int(p.c.table[1, 0])] = 0
    p.c.table[1, 1] = 99
    a = dev([1])
    si.si_cache_trim(p.c.desc, a.data_ptr(), 1, None, p.stream)
    torch.cuda.synchronize()
    assert int(p.c.status.item()) == si.SI_CACHE_BAD_PAGE and int(p.c.refs.min()) >= 0 and p.c.table[1].tolist() == [-1] * 12


def test_packing_in_place_and_into_another_pool():
    for seed in range(3):
        p = Pool(n_pages=50, seed=seed)
        p.extend([0, 1, 2, 3, 4], [32 * 5, 32 * 3 + 1, 200, 9, 100])
        p.fork([2], [5])
        p.trim([0, 1, 4], [32 * seed, 0, 33])
        place, m = p.books.compact()
        to = Cache(BF, m + 2 * seed, 32, 8, 12, 2, 1, 64, None, seed + 9)
        to.refs.fill_(5)
        to.table.fill_(77)
        before = to.bits().reshape(m + 2 * seed, -1).copy()
        used = torch.full((1,), -1, dtype=torch.int32, device="cuda")
        si.si_cache_compact(p.c.desc, to.desc, used.data_ptr(), p.stream)
        p.check()
        assert int(used.item()) == m
        b = p.books
        assert np.array_equal(to.table.cpu().numpy(), np.where(b.table >= 0, place[np.maximum(b.table, 0)], -1))
        assert np.array_equal(to.lens.cpu().numpy(), b.lens)
        refs = np.zeros(m + 2 * seed, np.int32)
        bits = to.bits().reshape(m + 2 * seed, -1)
        for q in range(len(place)):
            if place[q] >= 0:
                refs[place[q]] = b.refs[q]
                assert np.array_equal(bits[place[q]], p.original[b.content[q]])
        assert np.array_equal(to.refs.cpu().numpy(), refs)
        assert np.array_equal(bits[m:], before[m:])
        p.compact_in_place()
        p.compact_in_place()
        p.extend([6, 1], [100, 40])


def test_a_pool_that_is_too_small_is_not_packed_into():
    p = Pool()
    p.extend([0, 1], [100, 40])
    to = Cache(BF, 5, 32, 8, 12, 2, 1, 64, None, 3)
    before, used = to.bits().copy(), torch.zeros(1, dtype=torch.int32, device="cuda")
    si.si_cache_compact(p.c.desc, to.desc, used.data_ptr(), p.stream)
    torch.cuda.synchronize()
    assert int(p.c.status.item()) == si.SI_CACHE_NO_PAGES and int(used.item()) == 6
    assert np.array_equal(to.bits(), before) and int(to.lens.sum()) == 0 and bool((to.table == -1).all()) and int(to.refs.sum()) == 0


@pytest.mark.parametrize("n_pages,page,kv_heads,d,n_layers", [(20000, 32, 1, 64, 1), (30, 256, 4, 256, 3)])
def test_large_pools_and_large_pages(n_pages, page, kv_heads, d, n_layers):
    """More pages than one sweep of the reference counts; pages of more than one piece to copy."""
    p = Pool(n_pages=n_pages, page=page, kv_heads=kv_heads, d=d, n_layers=n_layers, n_seqs=16, max_pages=3000)
    n = n_pages // 4
    p.extend([0, 1, 2], [n * page - 3, n * page, page])
    p.fork([0], [3])
    p.trim([0, 3], [page + 1, 5])
    p.compact_in_place()
    p.extend([4, 5], [page * (n // 2), page * 2])


def test_long_lists():
    n = si.SI_CACHE_MAX_LIST
    p = Pool(n_pages=3 * n, n_seqs=n + 5, max_pages=3)
    r = random.Random(1)
    p.extend(r.sample(range(n + 5), n), [r.choice([0, 1, 31, 32, 33, 50]) for _ in range(n)])
    p.trim(r.sample(range(n + 5), n // 2))
    empty = [int(s) for s in np.flatnonzero(p.books.lens == 0)]
    parents = [int(s) for s in np.flatnonzero(p.books.lens > 0)]
    p.fork([r.choice(parents[:40]) for _ in empty], empty)
    p.extend(empty, [1] * len(empty), uniform=True)


@pytest.mark.parametrize("seed", range(6))
def test_random_calls(seed):
    r = random.Random(seed)
    p = Pool(r.choice([BF, F8]), n_pages=r.choice([20, 33]), n_seqs=9, max_pages=6, seed=seed)
    page = p.c.page
    for _ in range(40):
        seqs = r.sample(range(9), r.randint(1, 9))
        op = r.choice(["extend", "extend", "trim", "fork", "compact"])
        if op == "extend":
            if r.random() < 0.3:
                p.extend(seqs, [r.randint(0, 3)] * len(seqs), uniform=True, capacity=40)
            else:
                p.extend(seqs, [r.choice([0, 1, 2, page - 1, page, page + 5]) for _ in seqs], capacity=r.choice([60, 600]))
        elif op == "trim":
            p.trim(seqs, [r.randint(0, int(p.books.lens[s]) + (r.random() < 0.05)) for s in seqs] if r.random() < 0.8 else None)
        elif op == "fork":
            children = [s for s in seqs if p.books.lens[s] == 0]
            parents = [s for s in range(9) if s not in children]
            if children and parents:
                p.fork([r.choice(parents) for _ in children], children)
        else:
            p.compact_in_place()


def test_a_recorded_step_of_extend_and_trim():
    p = Pool(n_pages=60)
    p.extend([0, 1, 2], [10, 31, 64])
    seqs, keep = dev([0, 1, 2]), dev([0, 0, 0])
    seq, pos = (torch.zeros(8, dtype=torch.int32, device="cuda") for _ in range(2))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s = torch.cuda.current_stream().cuda_stream
        si.si_cache_trim(p.c.desc, seqs.data_ptr(), 3, keep.data_ptr(), s)
        si.si_cache_extend(p.c.desc, seqs.data_ptr(), 3, None, 2, seq.data_ptr(), pos.data_ptr(), 8, s)
    for step in range(5):
        k = [int(x) - (i + step) % 2 for i, x in enumerate(p.books.lens[:3])]
        keep.copy_(torch.tensor(k, dtype=torch.int32))
        assert p.books.trim([0, 1, 2], k) == 0
        want, status = p.books.extend([0, 1, 2], [2, 2, 2], 8)
        graph.replay()
        p.check(status)
        assert list(zip(seq.tolist(), pos.tolist())) == want
        p.extend([4], [step + 1])


def test_empty_lists():
    p = Pool()
    for f in (lambda: si.si_cache_trim(p.c.desc, None, 0), lambda: si.si_cache_extend(p.c.desc, None, 0, None, 1, None, None, 0), lambda: si.si_cache_fork(p.c.desc, None, None, 0)):
        f()
    p.check()
    p.compact_in_place()
