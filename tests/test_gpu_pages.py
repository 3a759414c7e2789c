"""Who holds which page, against lists of pages (tests/pages_ref.py): tables, lengths, counts and the pool's bits have to be equal."""
import random

import pytest
import torch

import pages_ref as R
from paper_2504_10724_amd import capi as ee
from paper_2504_10724_amd import paged as P

pytestmark = pytest.mark.gpu


def _i32(v, device="cuda"):
    return torch.tensor(v, dtype=torch.int32, device=device)


class Pair:
    """a cache with its bookkeeping on the device, and the same in lists"""

    def __init__(self, n_pages, page=32, layers=2, hkv=2, hd=64, dtype="f32", max_seqs=4096, values=True):
        self.kv = P.PagedCache(layers, n_pages, hkv, hd, page, dtype)
        pool = None
        if values:
            self.kv.pool.copy_(torch.arange(self.kv.pool.numel(), device="cuda") % 65521 if dtype == "f32"
                               else torch.randint(-128, 128, self.kv.pool.shape, device="cuda"))
            pool = self.kv.pool.cpu().view(layers, n_pages, hkv, 2 if dtype == "f32" else 1, page // 32, -1)
        self.pages, self.book = P.Pages(self.kv, max_seqs), R.Book(n_pages, page, pool)
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.tables = []

    def table(self, n, width):
        t = (P.PageTable(self.kv, n, width), self.book.table(n, width))
        self.tables.append(t)
        return t

    def grow(self, t, new=None):
        self.pages.grow(t[0], None if new is None else _i32(new), status=self.status)
        self.book.grow(t[1], new)

    def fork(self, t, parent, source=None, keep=None, group=0, rows=()):
        dev = [x.cuda() for x in rows]
        self.pages.fork(t[0], _i32(parent), source=None if source is None else source[0], keep=None if keep is None else _i32(keep), group=group,
                        rows=dev, status=self.status)
        self.book.fork(t[1], parent, None if source is None else source[1], keep, group, rows)
        for a, b in zip(dev, rows):
            assert torch.equal(a.cpu(), b)

    def compact(self):
        self.pages.compact(*(t[0] for t in self.tables))
        self.book.compact()

    def check(self, what=""):
        torch.cuda.synchronize()
        for i, (dev, ref) in enumerate(self.tables):
            assert dev.kv_len.tolist() == ref.len, (what, i)
            assert dev.pages.tolist() == ref.entries(), (what, i)
        refs = self.book.refs()
        assert self.pages.refs.tolist() == refs, what
        assert int(self.status.item()) == self.book.status, what
        if self.book.pool is not None:
            assert torch.equal(self.kv.pool.cpu(), self.book.pool.reshape(-1)), what
        return sum(r == 0 for r in refs)


@pytest.mark.parametrize("dtype,hkv,hd,page,layers", [("bf16", 2, 64, 32, 3), ("bf16", 1, 128, 96, 1), ("bf16", 3, 256, 64, 2), ("f32", 2, 4, 32, 1),
                                                      ("f32", 1, 84, 128, 2), ("f32", 3, 256, 64, 3)])
def test_a_long_run_of_calls(dtype, hkv, hd, page, layers):
    """beams that fork, requests that come, are cut and end, pages that run out, tables that are compacted"""
    print(f"[case] run {dtype} {hkv} heads of {hd}, pages of {page}", flush=True)
    r = random.Random(hd + page)
    c = Pair(20, page, layers, hkv, hd, dtype, max_seqs=12)
    t, store = c.table(12, 7), c.table(3, 5)
    c.grow(store, [3 * page + 5, 17, 2 * page])
    c.check("store")
    short = 0
    for step in range(60):
        what = r.choice(("grow", "grow", "grow", "one", "fork", "group", "take", "cut", "end", "compact"))
        if what == "grow":
            c.grow(t, [r.choice((0, 0, 1, 1, 2, r.randint(0, 2 * page))) for _ in range(12)])
        elif what == "one":
            c.grow(t)
        elif what == "fork":
            c.fork(t, [r.randrange(12) for _ in range(12)])
        elif what == "group":
            c.fork(t, [r.randrange(-1 if r.random() < 0.2 else 0, 4) for _ in range(12)], group=4)
        elif what == "take":
            c.fork(t, [r.randrange(-1, 3) for _ in range(12)], source=store, keep=[r.randint(0, 4 * page) for _ in range(12)])
        elif what == "cut":
            c.fork(t, list(range(12)), keep=[r.randint(0, 5 * page) for _ in range(12)])
        elif what == "end":
            c.fork(t, [i if r.random() < 0.6 else -1 for i in range(12)])
        else:
            c.compact()
        c.check((step, what))
        short += c.book.status >> 2 & 1
        c.status.zero_()
        c.book.status = 0
    assert short > 0
    c.fork(t, [-1] * 12)
    c.fork(store, [-1] * 3)
    assert c.check("end") == 20


@pytest.mark.parametrize("length", [1, 31, 32, 33, 63, 64])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_who_copies_a_shared_page(dtype, length):
    """all that hold it write: the first keeps it; one that does not write: all writers copy; a whole page is not written"""
    print(f"[case] writers {dtype} {length}", flush=True)
    c = Pair(40, 64, dtype=dtype)
    t = c.table(6, 3)
    c.grow(t, [length, 0, 0, 0, 0, 0])
    c.fork(t, [0, 0, 0, 0, -1, -1])
    c.grow(t, [0, 1, 0, 2, 0, 40])                           # two of four write
    c.check("two")
    c.grow(t, [1, 0, 1, 0, 0, 0])                            # the rest, who have it to themselves
    c.check("rest")
    c.fork(t, [1, 1, 1, 1, 1, -1])
    c.grow(t)                                                # all of them, and an empty row
    c.check("all")
    c.fork(t, [5, 4, 3, 2, 1, 0], keep=[1, 2, 3, 200, 0, 5])
    c.grow(t, [1, 64, 65, 3, 2, 100])
    c.check("other lengths")


def test_too_few_pages_change_nothing():
    print("[case] short", flush=True)
    c = Pair(5, 32, dtype="bf16")
    t = c.table(3, 4)
    c.grow(t, [33, 32, 10])                                  # 2 + 1 + 1 of 5
    c.check("first")
    c.grow(t, [32, 32, 10])                                  # two needed, one left
    c.check("short")
    assert c.book.status == 4
    c.grow(t, [31, 1, 22])                                   # exactly one
    assert c.check("last one") == 0
    c.grow(t, [0, 0, 0])
    c.check("none needed")
    c.fork(t, [0, 0, 0])
    c.check("forked")
    c.grow(t, [1, 0, 0])
    c.check("a page of its own")


def test_rows_outside_their_figures_stay():
    print("[case] figures", flush=True)
    c = Pair(30, 32)
    t = c.table(5, 2)
    c.grow(t, [40, 64, 1, 0, 65])                            # 65 positions do not fit two pages
    assert c.check("beyond") == 25 and c.book.status == 8
    c.grow(t, [-1, 1, 5, 2 ** 31 - 1, 64])
    c.check("negative")
    c.book.status = 0
    c.status.zero_()
    c.fork(t, [1, 5, -2, 2 ** 31 - 1, -2 ** 31])
    assert c.check("parents") and c.book.status == 8
    c.fork(t, [1, 2, 3, 4, 0], keep=[-1, 3, 2 ** 31 - 1, -2 ** 31, 33])
    c.check("keep")
    c.fork(t, [0, 1, 2, 3, 4], group=1)                      # of groups of one only parent 0 is a row
    c.check("groups of one")
    # a page number that is none, where the row's last positions should be; lengths that are none
    c2 = Pair(30, 32)
    t2 = c2.table(4, 2)
    c2.grow(t2, [5, 5, 5, 32])
    t2[0].pages[0, 0], t2[0].pages[1, 0] = 30, -1
    t2[0].kv_len[2] = -5
    before = t2[0].pages.clone()
    c2.pages.grow(t2[0], status=c2.status)
    assert int(c2.status.item()) == 9 and t2[0].kv_len.tolist() == [5, 5, -5, 33]
    before[3, 1] = 4
    assert torch.equal(t2[0].pages, before)


@pytest.mark.parametrize("n,group", [(1, 0), (7, 0), (64, 1), (60, 3), (128, 64), (300, 0), (2000, 1000), (4096, 0), (4096, 4096)])
@pytest.mark.parametrize("width", [1, 5, 70])
def test_forks_in_place(n, group, width):
    """every row a child of any other of its group, cut, with states of several widths"""
    print(f"[case] fork {n} rows in groups of {group}, width {width}", flush=True)
    r, page = random.Random(n + width), 32
    c = Pair(min(n * width, 6000) + 1, page, layers=1, hkv=1, hd=4, values=False)
    t = c.table(n, width)
    new, left = [], c.book.n - 1
    for _ in range(n):
        k = r.randint(0, min(width, left))
        left -= k
        new.append(max(0, k * page - r.randrange(page)))
    c.grow(t, new)
    c.check("grown")
    lim = group or n
    gen = torch.Generator().manual_seed(n)
    wide = torch.randint(0, 255, (n, 200), generator=gen, dtype=torch.uint8)
    for turn in range(2):
        rows = [torch.randint(0, 2 ** 30, (n, 9), generator=gen, dtype=torch.int32), torch.randn((n, 4, 20), generator=gen),
                torch.randint(0, 255, (n, 3), generator=gen, dtype=torch.uint8), torch.randn((n, 0), generator=gen), torch.randn(n, generator=gen).double()]
        keep = [r.randint(0, width * page) for _ in range(n)] if turn else None
        c.fork(t, [r.randrange(-1, lim) for _ in range(n)], keep=keep, group=group, rows=rows)
        c.check(("forked", turn))
    # rows inside wider ones: what lies beside them stays
    dev, parent = wide.cuda(), [r.randrange(lim) for _ in range(n)]
    c.pages.fork(t[0], _i32(parent), group=group, rows=[dev[:, 3:100]])
    want = wide.clone()
    at = torch.tensor([p + (i // group * group if group else 0) for i, p in enumerate(parent)])
    want[:, 3:100] = wide[at, 3:100]
    assert torch.equal(dev.cpu(), want)


def test_forks_of_more_rows_than_grow():
    """16384 rows from another table, in groups of 4096 among each other"""
    print("[case] fork 16384", flush=True)
    n = 16384
    c = Pair(50, 32, layers=1, hkv=1, hd=4, values=False)
    store, t = c.table(20, 2), c.table(n, 3)
    r = random.Random(3)
    c.grow(store, [r.randint(1, 64) for _ in range(20)])
    c.fork(t, [r.randrange(-1, 20) for _ in range(n)], source=store)
    c.check("taken")
    c.fork(t, [r.randrange(-1, 4096) for _ in range(n)], group=4096, rows=[torch.randint(0, 99, (n, 8), dtype=torch.int32)],
           keep=[r.randint(0, 70) for _ in range(n)])
    c.check("forked")
    for call in (lambda: c.pages.grow(t[0]), lambda: c.pages.fork(t[0], _i32([0] * n))):
        with pytest.raises(ee.EEError):
            call()


@pytest.mark.parametrize("n,n_pages", [(1, 1), (3, 32), (700, 5000), (1024, 9000), (1025, 9000), (4096, 40000)])
def test_many_rows_and_pages(n, n_pages):
    """rows of many lengths among more free pages than are looked at at a time, some rows sharing"""
    print(f"[case] grow {n} rows, {n_pages} pages", flush=True)
    r, page = random.Random(n), 32
    width = max(1, 2 * n_pages // n) if n < 100 else 30
    c = Pair(n_pages, page, layers=1, hkv=1, hd=4, values=n <= 700)
    t = c.table(n, width)
    most = n_pages // n // 2 * page
    c.grow(t, [r.randint(0, max(1, most)) for _ in range(n)])
    c.check("first")
    c.fork(t, [r.randrange(n) if r.random() < 0.3 else i if r.random() < 0.7 else -1 for i in range(n)])
    c.check("forked")
    c.grow(t, [r.choice((0, 1, 1, 33)) for _ in range(n)])
    c.check("second")
    c.compact()
    c.check("compacted")
    c.grow(t)
    c.check("third")
    c.fork(t, [i if i % 7 == 0 else -1 for i in range(n)])
    c.compact()
    c.check("compacted again")


def test_a_row_that_needs_thousands_of_pages():
    print("[case] one long row", flush=True)
    c = Pair(20000, 32, layers=1, hkv=1, hd=4, values=False)
    t = c.table(3, 19000)
    c.grow(t, [32 * 9 + 1, 0, 5])
    c.grow(t, [0, 32 * 18000 + 7, 32])
    c.check("grown")
    c.fork(t, [1, -1, 1], keep=[32 * 17000 + 1, 0, 2 ** 31 - 1])
    c.check("forked")
    c.grow(t, [1, 0, 32 * 500])
    c.check("again")
    c.fork(t, [-1, 1, 2])
    c.compact()
    c.check("compacted")


def test_free_pages_far_behind():
    """a pool of more words of free bits than are looked at at a time, full but for its end and some pages on the way"""
    print("[case] almost full", flush=True)
    n_pages = 150000
    c = Pair(n_pages, 32, layers=1, hkv=1, hd=4, values=False)
    t = c.table(4, n_pages)
    c.grow(t, [32 * 70000, 32 * 3, 32 * (n_pages - 70000 - 20), 0])
    assert c.check("full") == 17
    c.grow(t, [0, 0, 0, 32 * 17])
    assert c.check("none left") == 0
    c.fork(t, [0, -1, 2, 3])
    c.grow(t, [1, 0, 0, 64])
    assert c.check("three in the middle") == 0
    c.fork(t, [0, 1, 2, 3], keep=[32 * 40000, 0, 2 ** 30, 32 * 5])
    c.grow(t, [5, 32 * 100, 0, 7])
    c.check("again")
    c.compact()
    c.check("compacted")


@pytest.mark.parametrize("dtype,hkv,hd,page", [("f32", 1, 4, 32), ("bf16", 3, 96, 96), ("f32", 2, 252, 64), ("bf16", 5, 128, 256)])
def test_copies_between_pools(dtype, hkv, hd, page):
    """pages out of order, into a pool of another size; pages outside either pool are left out"""
    print(f"[case] copy {dtype} {hkv} {hd} {page}", flush=True)
    a, b = P.PagedCache(3, 9, hkv, hd, page, dtype), P.PagedCache(3, 14, hkv, hd, page, dtype)
    for x in (a, b):
        x.pool.copy_(torch.randint(-128, 128, x.pool.shape, device="cuda"))
    want = b.pool.clone().view(3, 14, -1)
    src, dst = [8, 0, 3, 4, 9, 2, -1, 1], [0, 13, 5, 6, 1, 14, 2, -1]
    for i, j in zip(src, dst):
        if 0 <= i < 9 and 0 <= j < 14:
            want[:, j] = a.pool.view(3, 9, -1)[:, i]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    P.copy_pages(a, b, _i32(src[:4]), _i32(dst[:4]), status=status)
    assert int(status.item()) == 0 and torch.equal(b.pool.view(3, 14, -1), want)
    P.copy_pages(a, b, _i32(src), _i32(dst), status=status)
    assert int(status.item()) == 1 and torch.equal(b.pool.view(3, 14, -1), want)
    P.copy_pages(a, a, _i32([8, 7]), _i32([1, 0]))           # inside one pool
    whole = a.pool.view(3, 9, -1)
    assert torch.equal(whole[:, 1], whole[:, 8]) and torch.equal(whole[:, 0], whole[:, 7])
    P.copy_pages(a, b, _i32([]), _i32([]))


def test_pages_beyond_4_gb():
    """addresses past 32 bits: the last pages of a pool of more than 6 GB are copied, shared, and moved"""
    print("[case] large pool", flush=True)
    kv = P.PagedCache(1, 100, 32, 128, 4096, "bf16")
    assert kv.pool.nbytes > 6e9
    kv.pool.view(100, -1)[:] = torch.arange(100, device="cuda", dtype=torch.bfloat16)[:, None]
    P.copy_pages(kv, kv, _i32([97]), _i32([3]))
    assert (kv.pool.view(100, -1)[3] == 97).all()
    pages, t = P.Pages(kv, 3), P.PageTable(kv, 3, 99)
    pages.grow(t, _i32([98 * 4096, 33, 0]))
    assert t.pages[1, 0] == 98
    pages.fork(t, _i32([0, 1, 1]))
    pages.grow(t)                                            # row 2 copies page 98 to 99; row 0 finds none: all or nothing
    assert t.kv_len.tolist() == [98 * 4096, 33, 33]
    pages.grow(t, _i32([0, 1, 1]))
    assert t.pages[2, 0] == 99 and t.pages[1, 0] == 98
    a = kv.pool.view(100, 32, 128, -1)
    assert (a[99, :, :2] == 98).all() and (a[99, :, 2:] == 99).all()       # two groups of 32 positions of each head
    pages.fork(t, _i32([-1, 1, 2]))
    pages.compact(t)
    assert t.pages[:, 0].tolist() == [-1, 0, 1] and (a[0] == 98).all() and (a[1, :, :2] == 98).all() and (a[1, :, 2:] == 99).all()


def test_a_reset_and_other_streams():
    """a run of calls on a stream of its own while another one is busy"""
    print("[case] streams", flush=True)
    c = Pair(30, 32, dtype="bf16")
    t = c.table(4, 5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    busy = torch.zeros(1 << 26, device="cuda")
    with torch.cuda.stream(side):
        for _ in range(20):
            busy.add_(1.0)
        c.grow(t, [40, 0, 0, 3])
        c.fork(t, [0, 0, 0, 3])
        c.grow(t)
    side.synchronize()
    c.check("side")
    c.pages.reset()
    assert not c.pages.refs.any()
    t[0].pages.fill_(-1)
    t[0].kv_len.zero_()
    c.book.tables[0].rows, c.book.tables[0].len = [[], [], [], []], [0, 0, 0, 0]
    c.grow(t, [1, 2, 3, 4])
    c.check("after")


def test_refusals():
    print("[case] refusals", flush=True)
    c = Pair(10, 32)
    t, other = P.PageTable(c.kv, 4, 3), P.PageTable(c.kv, 4, 3)
    parent, x = _i32([0, 1, 2, 3]), torch.zeros(4, 8, device="cuda")
    far = P.PageTable(c.kv, 4, 3)
    far.device += 1
    bad = [lambda: c.pages.grow(t, parent.cpu()), lambda: c.pages.grow(t, parent.long()), lambda: c.pages.grow(t, parent[:3]), lambda: c.pages.grow(far),
           lambda: c.pages.grow(t, status=parent), lambda: c.pages.fork(t, parent.cpu()), lambda: c.pages.fork(t, parent[:2]),
           lambda: c.pages.fork(t, parent, keep=parent[:1]), lambda: c.pages.fork(t, parent, group=3), lambda: c.pages.fork(t, parent, group=-1),
           lambda: c.pages.fork(t, parent, group=2 ** 32), lambda: c.pages.fork(t, parent, source=far), lambda: c.pages.fork(far, parent),
           lambda: c.pages.fork(t, parent, source=P.PageTable(c.kv, 4, 4)), lambda: c.pages.fork(t, parent, source=P.PageTable(c.kv, 8, 3), group=4),
           lambda: c.pages.fork(t, parent, source=other, rows=[x]), lambda: c.pages.fork(t, parent, rows=[x.cpu()]), lambda: c.pages.fork(t, parent, rows=[x[:3]]),
           lambda: c.pages.fork(t, parent, rows=[x.t().contiguous().t()]), lambda: c.pages.fork(t, parent, rows=[x[:1].expand(4, 8)]),
           lambda: c.pages.fork(t, parent, rows=[x, x]), lambda: c.pages.fork(t, parent, rows=[torch.zeros(4, k + 1, device="cuda") for k in range(9)]),
           lambda: c.pages.fork(t, t.kv_len), lambda: c.pages.fork(t, parent, keep=t.kv_len), lambda: c.pages.fork(t, parent, rows=[parent]),
           lambda: c.pages.fork(t, parent, rows=[t.kv_len]), lambda: c.pages.fork(t, parent, rows=[t.pages]),
           lambda: c.pages.fork(t, parent, rows=[x.clone().requires_grad_()]), lambda: c.pages.compact(t, far), lambda: c.pages.compact(t, t),
           lambda: c.pages.compact(*(P.PageTable(c.kv, 1, 1) for _ in range(9))), lambda: P.Pages(c.kv, 0), lambda: P.Pages(c.kv, 4097),
           lambda: P.Pages(c.kv, 2 ** 32 + 1), lambda: P.PageTable(c.kv, -1, 3), lambda: P.PageTable(c.kv, 2 ** 32, 3),
           lambda: P.copy_pages(c.kv, P.PagedCache(2, 4, 2, 64, 64, "f32"), parent, parent), lambda: P.copy_pages(c.kv, c.kv, parent, parent[:3]),
           lambda: P.copy_pages(c.kv, c.kv, parent.cpu(), parent.cpu())]
    for i, call in enumerate(bad):
        print(f"[refusal] {i}", flush=True)
        with pytest.raises(ee.EEError):
            call()
    small = P.Pages(c.kv, 3)
    with pytest.raises(ee.EEError):
        small.grow(t)                                        # four rows
    small.close()
    with pytest.raises(ee.EEError):
        small.reset()
    c.kv.close()
    for call in (lambda: c.pages.grow(t), lambda: c.pages.fork(t, parent), lambda: c.pages.compact(t), lambda: c.pages.reset(), lambda: P.Pages(c.kv, 3)):
        with pytest.raises(ee.EEError):
            call()
    assert not t.kv_len.any() and (t.pages == -1).all()


@pytest.mark.parametrize("n", [3, 1500])
def test_rows_grow_by_their_own_lengths(n):
    """the lengths are read as new positions and written as lengths in one call"""
    a = Pair(6 * n, values=False)
    t = a.table(n, 4)
    a.grow(t, [1 + i % 40 for i in range(n)])
    for _ in range(2):                                       # rows that would pass the table's end stay
        a.pages.grow(t[0], t[0].kv_len, status=a.status)
        a.book.grow(t[1], list(t[1].len))
        a.check()


def test_states_beside_each_other():
    """columns of one tensor as states of their own: their rows lie between each other's, not in them; one column more is refused"""
    print("[case] states beside each other", flush=True)
    c = Pair(10, 32)
    t = c.table(6, 2)
    x = torch.arange(6 * 40, dtype=torch.int32, device="cuda").view(6, 40)
    want, parent = x.clone(), [3, 3, 0, 1, 5, 2]
    want[:, 1:9], want[:, 12:], want[:, 9] = x[parent, 1:9], x[parent, 12:], x[parent, 9]
    c.pages.fork(t[0], _i32(parent), rows=[x[:, 1:9], x[:, 12:], x[:, 9:10]])
    assert torch.equal(x, want)
    for rows in ([x[:, :9], x[:, 8:]], [x[:, 8:9], x], [x.view(-1)[4:40].view(6, 6), x[:, 39:]], [x[:, 3], x[:, 3:]]):
        with pytest.raises(ee.EEError):
            c.pages.fork(t[0], _i32(parent), rows=rows)
    assert torch.equal(x, want)


def test_tangents_of_states_are_not_lost():
    print("[case] tangents", flush=True)
    from torch.autograd import forward_ad
    c = Pair(10, 32)
    t, x = c.table(4, 2), torch.arange(8.0, device="cuda").view(4, 2)
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(x, torch.ones_like(x))
        for _ in range(2):
            with pytest.raises(ee.EEError, match="gradient"):
                c.pages.fork(t[0], _i32([1, 0, 2, 2]), rows=[dual])
            with torch.no_grad(), pytest.raises(ee.EEError, match="gradient"):
                c.pages.fork(t[0], _i32([1, 0, 2, 2]), rows=[dual])
        c.pages.fork(t[0], _i32([1, 0, 2, 2]), rows=[dual.detach()])
    assert x.tolist() == [[2.0, 3.0], [0.0, 1.0], [4.0, 5.0], [4.0, 5.0]]
