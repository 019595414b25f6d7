"""The book of a cache's pages, and copies of pages, against the definition."""
import numpy as np
import pytest
import torch

import paper_2608_09160_amd as qkn
from oracle import pages as O

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _i32(x):
    return torch.tensor(list(x), dtype=torch.int32, device=DEV)


def _ints(t):
    return t.cpu().tolist()


class Both:
    """A book on the device and the oracle's, the same after every call."""

    def __init__(self, pages, rows, max_tokens, page_size):
        self.dev = qkn.PageBook.empty(pages, rows, max_tokens, page_size, DEV)
        self.ref = O.Book(*(t.cpu().numpy() for t in (self.dev.refs, self.dev.table, self.dev.kv_len)), page_size)

    def same(self, check=True):
        torch.cuda.synchronize()
        assert _ints(self.dev.refs) == self.ref.refs.tolist() and _ints(self.dev.kv_len) == self.ref.kv_len.tolist()
        got = O.Book(*(t.cpu().numpy() for t in (self.dev.refs, self.dev.table, self.dev.kv_len)), self.ref.page)
        assert got.held() == self.ref.held()
        if check:
            got.check()

    def grow(self, counts, which=None, T=None):
        T = sum(max(c, 0) for c in counts) if T is None else T
        slots, pos = torch.full((T,), 77, dtype=torch.int64, device=DEV), torch.full((T,), 77, dtype=torch.int32, device=DEV)
        done = qkn.qkn_pages_grow(self.dev, _i32(counts), None if which is None else _i32(which), slots, pos)
        want = self.ref.grow(counts, which, T)
        self.same()
        assert [_ints(done), _ints(slots), _ints(pos)] == [list(map(int, w)) for w in want]
        return want

    def fork(self, parents, to):
        n = len(to)
        call = qkn.PreparedPagesFork(self.dev, _i32(parents), _i32(to), _i32([77] * n), _i32([77] * n), _i32([77] * n))
        call()
        want = self.ref.fork(parents, to)
        self.same()
        assert [_ints(call.done), _ints(call.src), _ints(call.dst)] == [list(map(int, w)) for w in want]
        return want

    def free(self, which):
        qkn.qkn_pages_free(self.dev, _i32(which))
        self.ref.free(which)
        self.same()

    def compact(self, n, out=False):
        src, dst = _i32([77] * n), _i32([77] * n)
        new = qkn.PageBook(torch.full_like(self.dev.refs, 99), torch.full_like(self.dev.table, 99), self.dev.kv_len,
                           self.dev.page_size) if out else None
        old = [t.clone() for t in (self.dev.refs, self.dev.table)]
        qkn.qkn_pages_compact(self.dev, src, dst, out=new)
        if out:
            assert torch.equal(old[0], self.dev.refs) and torch.equal(old[1], self.dev.table)
            self.dev = new
        want = self.ref.compact(n)
        self.same()
        assert [_ints(src), _ints(dst)] == [list(map(int, w)) for w in want]
        return want


def test_growing_step_by_step():
    b = Both(40, 4, 100, 16)
    b.grow([1, 0, 17, 32])
    b.grow([15, 16, 1, 1])
    b.grow([1, 1, 1, 1])
    b.grow([3, 50], [2, 0])
    b.grow([0, 0, 0, 0])


def test_refused_rows():
    b = Both(10, 6, 64, 16)
    b.grow([16, 16], [1, 3])
    b.grow([5, -1, 65, 64, 3, 2, 1], [0, 1, 2, 2, 9, -1, 1])  # 2 and 1 again: listed before
    b.grow([49, 48], [1, 3])  # a row's room
    assert b.ref.kv_len.tolist() == [5, 16, 0, 64, 0, 0]


def test_a_pool_that_does_not_suffice():
    b = Both(6, 5, 64, 16)
    b.grow([10, 40, 40, 6, 1])  # 1 + 3 pages; 3 more are not there, nor is one for the later rows
    assert b.ref.kv_len.tolist() == [10, 40, 0, 0, 0]
    b.grow([6, 8, 33, 16, 16])  # rows that need none are served whatever stands before them
    assert b.ref.kv_len.tolist() == [16, 48, 0, 0, 0]
    b.grow([0, 0, 33, 5, 0])
    b.grow([16, 1, 1])
    b.free([0])
    b.grow([1, 1, 1, 1, 1])
    b.fork([1, 1], [2, 3])
    b.fork([0, 4], [2, 3])


def test_tokens_of_the_list():
    b = Both(64, 5, 200, 16)
    b.grow([20, 0, 3, 40], [3, 0, 1, 2], T=100)  # more places than tokens
    b.grow([20, 5, 3, 40], [3, 0, 1, 2], T=30)   # fewer
    b.grow([1, 250, 2], [3, 0, 1])               # a refused row keeps its places
    b.grow([5, 5], T=0)
    done = qkn.qkn_pages_grow(b.dev, _i32([1, 1]))
    want = b.ref.grow([1, 1])
    b.same()
    assert _ints(done) == list(map(int, want[0]))
    pos = torch.zeros(2, dtype=torch.int32, device=DEV)
    qkn.qkn_pages_grow(b.dev, _i32([1, 1]), pos=pos)
    want = b.ref.grow([1, 1], T=2)
    b.same()
    assert _ints(pos) == list(map(int, want[2]))


@pytest.mark.parametrize("page", [1, 16, 64])
def test_forks(page):
    b = Both(200, 12, 5 * page + 3, page)
    b.grow([5 * page, 2 * page + page // 2, 1, 0][:4])
    b.fork([0, 1, 2, 3, 1], [4, 5, 6, 7, 8])
    b.fork([5, 5], [9, 10])          # a branch's branches
    b.grow([1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1])
    b.free([1, 0])
    b.fork([4, 4, 99, -1, 4, 2, 2], [0, 1, 1, 1, 12, -1, 2])  # outside the book, listed before, not empty
    b.free([5, 8, 4, 4, 77, -3])
    b.fork([9, 11], [11, 4])         # lengths are those before the call: 11 forks as an empty row
    b.free(range(12))
    assert not b.ref.refs.any()


def test_moving_pages_to_the_front():
    b = Both(50, 8, 160, 16)
    b.grow([100, 30, 160, 17, 1, 160, 90, 16])
    b.free([0, 2, 4])
    b.compact(2)     # as many as the lists hold
    b.compact(50, out=True)
    b.compact(50)    # nothing to move
    b.fork([1, 3, 3], [0, 2, 4])
    b.free([5, 7])
    b.compact(7)
    b.free(range(8))
    b.compact(5)
    b.compact(0)


def test_entries_past_a_rows_last_page_are_kept():
    b = Both(30, 3, 160, 16)
    b.grow([100, 30, 40])
    b.free([0])
    before = b.dev.table.clone()
    b.compact(30, out=True)
    past = torch.arange(10, device=DEV) >= (b.dev.kv_len[:, None] + 15) // 16
    assert torch.equal(b.dev.table[past], before[past])


@pytest.mark.parametrize("seed", range(12))
def test_random_calls(seed):
    rng = np.random.default_rng(seed)
    page = int(rng.choice([1, 16, 32]))
    rows, per = int(rng.integers(1, 40)), int(rng.integers(1, 20))
    b = Both(int(rng.integers(1, rows * per + 20)), rows, per * page, page)
    for _ in range(25):
        kind = rng.choice(["grow", "grow", "fork", "free", "compact"])
        n = int(rng.integers(1, rows + 1))
        which = rng.integers(-1, rows + 1, n).tolist()
        if kind == "grow":
            counts = rng.integers(-1, 3 * page + 2, n).tolist()
            b.grow(counts, which if rng.random() < 0.7 else None, T=int(rng.integers(0, 200)))
        elif kind == "fork":
            b.fork(rng.integers(-1, rows + 1, n).tolist(), which)
        elif kind == "free":
            b.free(which)
        else:
            b.compact(int(rng.integers(0, 30)), out=rng.random() < 0.5)


@pytest.mark.parametrize("pages", [16384, 16385, 70001])
def test_large_books(pages):
    """More pages than a pass over them takes, 1024 rows."""
    b = Both(pages, 1024, 1024, 16)
    rng = np.random.default_rng(pages)
    b.grow(rng.integers(0, 1025, 1024).tolist() if pages > 40000 else rng.integers(0, 200, 1024).tolist())
    b.free(rng.permutation(1024)[:600].tolist())
    b.grow(rng.integers(0, 100, 1024).tolist(), rng.permutation(1024).tolist())
    empty = np.flatnonzero(b.ref.kv_len == 0)
    b.fork(rng.permutation(1024)[:len(empty)].tolist(), empty.tolist())
    b.free(rng.permutation(1024)[:500].tolist())
    src, dst = (torch.empty(pages, dtype=torch.int32, device=DEV) for _ in range(2))
    qkn.qkn_pages_compact(b.dev, src, dst)
    used, free = np.flatnonzero(b.ref.refs), np.flatnonzero(b.ref.refs == 0)
    moves = int((used >= len(used)).sum())
    assert _ints(src) == used[::-1][:moves].tolist() + [-1] * (pages - moves)
    assert _ints(dst) == free[:moves].tolist() + [-1] * (pages - moves)
    got = O.Book(*(t.cpu().numpy() for t in (b.dev.refs, b.dev.table, b.dev.kv_len)), 16)
    got.check()
    where = dict(zip(used[::-1][:moves].tolist(), free[:moves].tolist()))
    assert got.held() == [[where.get(p, p) for p in row] for row in b.ref.held()]


@pytest.mark.parametrize("pages,every", [(5000, 1), (40000, 3), (70001, 7)])
def test_many_pages_at_once(pages, every):
    """More pages than one pass over the book finds, some passes with few or none; a row that does not get all of them."""
    b = Both(pages, 40, 1 << 14, 2)
    refs = np.ones(pages, np.int32)
    refs[::every] = 0
    refs[4096:8192] = 1  # a part without free pages
    refs[20000:37000] = 1
    b.dev.refs.copy_(torch.from_numpy(refs))
    b.ref.refs[:] = refs
    free = int((refs == 0).sum())
    counts = [2 * (free // 5) - 1, 0, 1, 2 * (free // 2), 3, 2 * free, 0, 1]
    counts = [min(c, 1 << 14) for c in counts]
    done = qkn.qkn_pages_grow(b.dev, _i32(counts))
    want = b.ref.grow(counts, None, 0)
    assert _ints(done) == [int(x) for x in want[0]]
    got = O.Book(*(t.cpu().numpy() for t in (b.dev.refs, b.dev.table, b.dev.kv_len)), 2)
    assert np.array_equal(got.refs, b.ref.refs) and np.array_equal(got.kv_len, b.ref.kv_len) and got.held() == b.ref.held()
    rows = list(range(8, 40))
    call = qkn.PreparedPagesFork(b.dev, _i32([0, 2] * 16), _i32(rows), _i32([77] * 32), _i32([77] * 32), _i32([77] * 32))
    call()
    want = b.ref.fork([0, 2] * 16, rows)
    assert [_ints(call.done), _ints(call.src), _ints(call.dst)] == [list(map(int, w)) for w in want]
    got = O.Book(*(t.cpu().numpy() for t in (b.dev.refs, b.dev.table, b.dev.kv_len)), 2)
    assert np.array_equal(got.refs, b.ref.refs) and np.array_equal(got.kv_len, b.ref.kv_len) and got.held() == b.ref.held()


def test_malformed_books_stay_inside_their_arrays():
    """Lengths and page numbers outside their ranges; what lies around the arrays keeps its values."""
    room = {n: torch.full((k + 64,), 1234, dtype=torch.int32, device=DEV) for n, k in (("refs", 8), ("table", 20), ("kv_len", 5))}
    view = {n: t[32:-32] for n, t in room.items()}
    book = qkn.PageBook(view["refs"], view["table"].view(5, 4), view["kv_len"], 16)
    src, dst = torch.full((40,), 1234, dtype=torch.int32, device=DEV), torch.full((40,), 1234, dtype=torch.int32, device=DEV)
    for lens in ([-5, 65, 1 << 30, -(1 << 31), 64], [64, 64, 1, 17, 0]):
        for entry in (-1, 8, 1 << 30, -(1 << 31), 3):
            for call in (lambda: qkn.qkn_pages_grow(book, _i32([3, 3, 3, 3, 3]), slots=torch.empty(15, dtype=torch.int64, device=DEV)),
                         lambda: qkn.PreparedPagesFork(book, _i32([0, 1, 2, 3, 4]), _i32([4, 3, 2, 1, 0]), src[16:21], dst[16:21])(),
                         lambda: qkn.qkn_pages_free(book, _i32([4, 3, 2, 1, 0])),
                         lambda: qkn.qkn_pages_compact(book, src[16:24], dst[16:24])):
                view["refs"].copy_(_i32([0, 1, 2, -3, 0, 1 << 30, 1, 0]))
                view["table"].fill_(entry)
                view["kv_len"].copy_(_i32(lens))
                call()
                torch.cuda.synchronize()
                for t in room.values():
                    assert (t[:32] == 1234).all() and (t[-32:] == 1234).all()
                for t in (src, dst):
                    assert (t[:16] == 1234).all() and (t[24:] == 1234).all()
        done = qkn.qkn_pages_grow(book, _i32([0, 0, 0, 0, 0]))
        torch.cuda.synchronize()
    view["kv_len"].copy_(_i32([-5, 65, 1 << 30, -(1 << 31), 64]))
    assert _ints(qkn.qkn_pages_grow(book, _i32([0] * 5))) == [-1, -1, -1, -1, 64]


def _pools(fmt, pages, heads, page, D, order, g):
    """A cache of random bytes and its pools as bytes."""
    def pool(width):
        shape = (pages, page, heads, width) if order == "rows first" else (pages, heads, page, width)
        x = torch.randint(0, 256, shape, dtype=torch.uint8, generator=g).to(DEV)
        return x.transpose(1, 2) if order == "rows first" else x
    if fmt == "fp4":
        pools = [pool(D // 2), pool(D // 2), pool(D // 32), pool(D // 32)]
        return qkn.KVCache4(*pools), pools
    pools = [pool(D * (2 if fmt == "bf16" else 1)) for _ in range(2)]
    return qkn.KVCache(*(p.view(torch.bfloat16) if fmt == "bf16" else p for p in pools)), pools


@pytest.mark.parametrize("order", ["heads first", "rows first"])
@pytest.mark.parametrize("fmt,heads,page,D,layers", [("bf16", 4, 16, 128, 3), ("fp8", 1, 64, 64, 30), ("fp4", 2, 16, 64, 21), ("bf16", 3, 4, 33, 1),
                                                     ("fp8", 3, 8, 13, 2), ("fp4", 1, 1, 32, 1), ("bf16", 8, 128, 256, 1)])
def test_copies(fmt, heads, page, D, layers, order):
    g = torch.Generator().manual_seed(D)
    n_pages = 40
    caches = [_pools(fmt, n_pages, heads, page, D, order, g) for _ in range(layers)]
    src = [3, -1, 39, 7, 5, 40, 1 << 30, 2, 0, 30, 7]
    dst = [10, 4, 11, 12, 5, 13, 14, -7, 40, 15, 16]
    want = [[p.clone() for p in pools] for _, pools in caches]
    for pools in want:
        for p in pools:
            for a, b in zip(src, dst):
                if 0 <= a < n_pages and 0 <= b < n_pages:
                    p[b] = p[a]
    qkn.qkn_pages_copy([c for c, _ in caches], _i32(src), _i32(dst))
    torch.cuda.synchronize()
    for (_, pools), ref in zip(caches, want):
        assert all(torch.equal(p, r) for p, r in zip(pools, ref))


def test_copies_leave_what_lies_between_rows():
    """Pools of one allocation, K and V in turn and gaps between rows; caches of other sizes in one call."""
    both = torch.randint(0, 256, (9, 2, 3, 16, 80), dtype=torch.uint8, device=DEV)
    few = torch.randint(0, 256, (5, 2, 3, 16, 64), dtype=torch.uint8, device=DEV)
    caches = [qkn.KVCache(both[:, 0, ..., :64], both[:, 1, ..., :64]), qkn.KVCache(few[:, 0], few[:, 1])]
    want, want_few = both.clone(), few.clone()
    want[1, ..., :64], want[8, ..., :64] = both[4, ..., :64], both[0, ..., :64]
    want_few[1] = few[4]  # page 8 is outside this one
    qkn.qkn_pages_copy(caches, _i32([4, 0, 2]), _i32([1, 8, 2]))
    torch.cuda.synchronize()
    assert torch.equal(both, want) and torch.equal(few, want_few)


def test_long_lists_with_few_pairs():
    g = torch.Generator().manual_seed(0)
    cache, pools = _pools("bf16", 5000, 2, 16, 64, "heads first", g)
    src, dst = (torch.full((100000,), -1, dtype=torch.int32, device=DEV) for _ in range(2))
    at = torch.randperm(100000, generator=g)[:2000].to(DEV)
    pages = torch.randperm(5000, generator=g)[:4000].to(DEV).int()
    src[at], dst[at] = pages[:2000], pages[2000:]
    want = [p.clone() for p in pools]
    for p in want:
        p[pages[2000:].long()] = p[pages[:2000].long()]
    qkn.qkn_pages_copy([cache], src, dst)
    torch.cuda.synchronize()
    assert all(torch.equal(p, w) for p, w in zip(pools, want))


def test_a_run_of_them_in_a_graph():
    """Branches dropped and forked, grown and moved to the front, replayed: each replay is the eager run's."""
    b = qkn.PageBook.empty(60, 6, 160, 16, DEV)
    g = torch.Generator().manual_seed(1)
    cache, pools = _pools("bf16", 60, 2, 16, 64, "heads first", g)
    src, dst = (torch.empty(30, dtype=torch.int32, device=DEV) for _ in range(2))
    slots, pos = torch.empty(4, dtype=torch.int64, device=DEV), torch.empty(4, dtype=torch.int32, device=DEV)
    fork = qkn.PreparedPagesFork(b, _i32([0, 1]), _i32([2, 3]))
    calls = [qkn.PreparedPagesFree(b, _i32([2, 3])), fork, qkn.PreparedPagesCopy([cache], fork.src, fork.dst),
             qkn.PreparedPagesGrow(b, _i32([1, 2, 1]), _i32([0, 2, 3]), slots, pos),
             qkn.PreparedPagesFree(b, _i32([4])),
             qkn.PreparedPagesGrow(b, _i32([30]), _i32([4])),
             qkn.PreparedPagesCompact(b, src, dst), qkn.PreparedPagesCopy([cache], src, dst)]
    qkn.qkn_pages_grow(b, _i32([40, 21, 5, 70, 100]))
    state = [b.refs, b.table, b.kv_len, *pools, slots, pos, src, dst, fork.src, fork.dst, fork.done]
    start = [t.clone() for t in state]
    eager = []
    for _ in range(4):
        for c in calls:
            c()
        torch.cuda.synchronize()
        eager.append([t.clone() for t in state])
    for t, s in zip(state, start):
        t.copy_(s)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        for c in calls:
            c()
    for t, s in zip(state, start):
        t.copy_(s)
    for want in eager:
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, w) for t, w in zip(state, want))
        O.Book(*(t.cpu().numpy() for t in (b.refs, b.table, b.kv_len)), 16).check()


def test_empty_calls():
    none, b = _i32([]), qkn.PageBook.empty(0, 0, 16, 16, DEV)
    qkn.qkn_pages_grow(b, none)
    qkn.qkn_pages_fork(b, none, none)
    qkn.qkn_pages_free(b, none)
    qkn.qkn_pages_compact(b, none, none)
    src, dst = _i32([5, 5]), _i32([5, 5])
    qkn.qkn_pages_compact(b, src, dst)
    assert _ints(src) == _ints(dst) == [-1, -1]
    qkn.qkn_pages_copy([], src, dst)
    b = qkn.PageBook.empty(0, 3, 64, 16, DEV)  # no pages at all
    assert _ints(qkn.qkn_pages_grow(b, _i32([1, 0, 2]))) == [-1, 0, -1]


def test_calls_on_a_given_stream():
    """Each call, and what it allocates, on the stream that it is given."""
    side = torch.cuda.Stream()
    b = Both(60, 6, 100, 16)
    cache, pools = _pools("bf16", 60, 2, 16, 64, "heads first", torch.Generator().manual_seed(2))
    counts, which, parents, to = _i32([40, 21, 5]), _i32([0, 1, 2]), _i32([0, 1, 1]), _i32([3, 4, 5])
    src, dst = (torch.empty(30, dtype=torch.int32, device=DEV) for _ in range(2))
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):  # another one is current
        qkn.qkn_pages_grow(b.dev, counts, which, stream=side)
        qkn.qkn_pages_fork(b.dev, parents, to, [cache], stream=side)
        qkn.qkn_pages_free(b.dev, which, stream=side)
        qkn.qkn_pages_compact(b.dev, src, dst, [cache], stream=side)
        qkn.qkn_pages_copy([cache], src, dst, stream=side)
    b.ref.grow([40, 21, 5], [0, 1, 2])
    b.ref.fork([0, 1, 1], [3, 4, 5])
    b.ref.free([0, 1, 2])
    want = b.ref.compact(30)
    b.same()
    assert [_ints(src), _ints(dst)] == [list(map(int, w)) for w in want]


@pytest.mark.parametrize("free", [3, 1023, 1026, 4099, 20011])
def test_what_a_refused_row_got_is_free_again(free):
    b = Both(free + 7, 4, free + 100, 1)
    b.grow([3, 0, 4, 0])
    b.grow([2, free, 1, 0])  # the second row is two pages short, and nothing is left for the third
    assert b.ref.kv_len.tolist() == [5, 0, 4, 0]
    b.grow([0, free - 2, 0, 0])  # all of them are there
    b.grow([1, 1, 0, 1])


def _least_us(call, before):
    spent = []
    for _ in range(4):
        before()
        torch.cuda.synchronize()
        begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        begin.record()
        call()
        end.record()
        torch.cuda.synchronize()
        spent.append(1e3 * begin.elapsed_time(end))
    return min(spent)


def test_a_refused_row_takes_no_longer_than_a_served_one():
    """A captured loop meets an empty pool on every replay: giving pages back is as wide as handing them out. Both read the
    pool once and write an entry a page; a thread that gave 65536 pages back by itself took 200 times the served call."""
    pages = 65536
    book = qkn.PageBook.empty(pages, 2, pages + 1, 1, DEV)
    served, refused = (qkn.PreparedPagesGrow(book, _i32([n, 0])) for n in (pages, pages + 1))

    def empty():
        book.refs.zero_()
        book.kv_len.zero_()

    there = _least_us(served, empty)
    assert _ints(served.done) == [pages, 0] and int(book.refs.sum()) == pages
    gone = _least_us(refused, empty)
    assert _ints(refused.done) == [-1, 0] and int(book.refs.sum()) == 0
    assert gone < 8 * there, (gone, there)


def test_all_rows_are_freed_without_a_list():
    b = Both(60, 6, 100, 16)
    b.grow([40, 21, 5, 0, 100, 16])
    b.fork([0], [3])
    qkn.qkn_pages_free(b.dev)
    b.ref.free(range(6))
    b.same()
    assert not b.ref.refs.any() and not b.ref.kv_len.any()
    b.grow([100] * 6)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    qkn.PreparedPagesFree(b.dev)(side)
    b.ref.free(range(6))
    b.same()
    qkn.qkn_pages_free(qkn.PageBook.empty(4, 0, 16, 16, DEV))
