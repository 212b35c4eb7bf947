"""The book of a paged cache (fork, reserve, trim, compact) against the same steps taken entry after entry in Python, number for number, and the
copying of pages byte for byte."""
import random

import pytest
import torch

import paper_2609_23153_b200 as sa
from test_gpu_cache import DEV, make_cache, same_bits

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Book:
    """Tables, counts and lengths as lists."""

    def __init__(self, table, refs, length, page):
        self.table, self.refs, self.len, self.page = [list(r) for r in table], list(refs), list(length), page

    def copy(self):
        return Book(self.table, self.refs, self.len, self.page)

    def there(self, e):
        return 0 <= e < len(self.refs)

    def fork(self, parent):
        B, columns = len(self.table), len(self.table[0])
        uses = [sum(p == b for p in parent) for b in range(B)]
        for b, row in enumerate(self.table):
            for e in row:
                if self.there(e):
                    self.refs[e] += uses[b] - 1
        self.table = [list(self.table[p]) if 0 <= p < B else [-1] * columns for p in parent]
        self.len = [self.len[p] if 0 <= p < B else 0 for p in parent]

    def reserve(self, new):
        P = self.page
        free = [p for p, r in enumerate(self.refs) if r == 0]
        fine = [0 <= n <= m <= len(self.table[0]) * P for n, m in zip(self.len, new)]
        active = [f and m > n for f, n, m in zip(fine, self.len, new)]
        tail = {b: self.table[b][self.len[b] // P] for b in range(len(new)) if active[b] and self.len[b] % P and self.there(self.table[b][self.len[b] // P])}
        writers = {}
        for b, e in tail.items():
            if self.refs[e] > 1:
                writers.setdefault(e, []).append(b)
        copies = {b for e, w in writers.items() for b in (w if len(w) != self.refs[e] else w[1:])}
        wanted = []
        for b in range(len(new)):
            if active[b]:
                wanted += [(b, self.len[b] // P)] if b in copies else []
                wanted += [(b, i) for i in range(-(-self.len[b] // P), -(-new[b] // P)) if self.table[b][i] == -1]
        src, dst = [-1] * len(new), [-1] * len(new)
        if len(wanted) > len(free):
            return src, dst, len(wanted) - len(free)
        for (b, i), p in zip(wanted, free):
            if b in copies and i == self.len[b] // P:
                src[b], dst[b] = self.table[b][i], p
                self.refs[src[b]] -= 1
            self.table[b][i] = p
            self.refs[p] = 1
        return src, dst, 0

    def trim(self, frame, window, sink):
        P = self.page
        for b, n in enumerate(self.len):
            if not 0 <= n <= len(self.table[b]) * P:
                continue
            lo = (n // frame - window + 1) * frame if window else 0
            for i, e in enumerate(self.table[b]):
                if i * P >= n or (i * P >= sink and (i + 1) * P <= lo):
                    if self.there(e):
                        self.refs[e] -= 1
                    self.table[b][i] = -1

    def compact(self):
        used = [r > 0 for r in self.refs]
        n = sum(used)
        src = [p for p in range(n, len(used)) if used[p]]
        dst = [p for p in range(n) if not used[p]]
        to = dict(zip(src, dst))
        self.table = [[to.get(e, e) if self.there(e) and used[e] else -1 for e in row] for row in self.table]
        for p, q in to.items():
            self.refs[q], self.refs[p] = self.refs[p], 0
        pad = [-1] * (len(used) // 2 - len(src))
        return src + pad, dst + pad


def make_book(rng, B, pages, page, columns, most, share=0.3, pinned=0.05):
    """Sequences of random lengths that share what they have in common with earlier ones, and pages that somebody else keeps as well."""
    order = list(range(pages))
    rng.shuffle(order)
    table, refs, length = [], [0] * pages, []
    for b in range(B):
        n = rng.choice((0, rng.randint(0, most), rng.randint(0, most), rng.randint(0, most) // page * page))
        row = [-1] * columns
        if b and rng.random() < share:
            other = rng.randrange(b)
            n = length[other] if rng.random() < 0.7 else min(n, length[other])
            row[:-(-n // page)] = table[other][:-(-n // page)]
        else:
            need = -(-n // page)
            if need > len(order):
                n, need = 0, 0
            for i in range(need):
                row[i] = order.pop()
        for e in row:
            if e >= 0:
                refs[e] += 1
        table.append(row)
        length.append(n)
    for p in range(pages):
        if rng.random() < pinned:
            refs[p] += 1
    return Book(table, refs, length, page)


SIZES = [
    # B, pages, page, columns, most tokens
    (1, 1, 16, 1, 16),
    (1, 2, 128, 3, 300),
    (3, 40, 16, 9, 100),
    (17, 600, 32, 40, 900),
    (64, 5000, 64, 130, 8000),
    (600, 3000, 16, 13, 150),
    (5, 70001, 16, 9000, 140000),
    (4096, 9000, 64, 5, 200),
]


def on_device(book):
    return ints(book.table), ints(book.len), ints(book.refs)


def workspace(pages):
    return torch.full((256 + (4 * pages + 255) // 256 * 256,), 0xA5, dtype=torch.uint8, device=DEV)


def same(got, want):
    return torch.equal(got.cpu(), torch.tensor(want, dtype=torch.int32))


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "-".join(str(x) for x in s))
@pytest.mark.parametrize("seed", [0, 1])
def test_fork(size, seed):
    rng = random.Random(seed)
    B, pages = size[0], size[1]
    book = make_book(rng, *size)
    for B_out in (B, max(1, B // 2), min(4096, 2 * B + 1)):
        parent = [rng.choice((-1, rng.randrange(B), rng.randrange(B), min(b, B - 1))) for b in range(B_out)]
        want = book.copy()
        want.fork(parent)
        table, length, refs = on_device(book)
        ws = workspace(pages)
        got = sa.pages_fork(table, length, refs, ints(parent), workspace=ws)
        assert sa.read_status(ws) == sa.OK
        assert same(got[0], want.table) and same(got[1], want.len) and same(got[2], want.refs)
        assert same(table, book.table) and same(refs, book.refs)                # the inputs stay
        sa.pages_fork(table, length, refs, ints(parent), refs_out=refs, check_status=True)
        assert same(refs, want.refs)


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "-".join(str(x) for x in s))
@pytest.mark.parametrize("seed", range(4))
def test_reserve(size, seed):
    rng = random.Random(100 + seed)
    B, pages, page, columns, most = size
    book = make_book(rng, *size, share=0.6)
    step = (1, page // 2, 3 * page, 40 * page)[seed]
    new = [min(n + rng.choice((0, 1, step, rng.randint(0, step))), columns * page) for n in book.len]
    if seed == 2:        # some have their pages already
        spare = [p for p, r in enumerate(book.refs) if r == 0]
        for b in range(0, B, 3):
            i = -(-book.len[b] // page)
            if i < columns and spare:
                book.table[b][i] = spare.pop(rng.randrange(len(spare)))
                book.refs[book.table[b][i]] = 1
    want = book.copy()
    src, dst, missing = want.reserve(new)
    table, length, refs = on_device(book)
    ws = workspace(pages)
    got = sa.pages_reserve(table, length, refs, ints(new), page, workspace=ws)
    assert sa.read_status(ws) == (sa.E_OUT_OF_PAGES if missing else sa.OK)
    assert int(ws.view(torch.int32)[1]) == missing
    assert same(got[0], want.table) and same(got[1], want.refs) and same(got[2], src) and same(got[3], dst)
    assert same(table, book.table) and same(refs, book.refs)
    sa.pages_reserve(table, length, refs, ints(new), page, page_table_out=table, refs_out=refs, workspace=ws)
    assert same(table, want.table) and same(refs, want.refs)
    if not missing:      # what has been reserved is not reserved again
        again = sa.pages_reserve(table, length, refs, ints(new), page, check_status=True)
        after = want.copy()
        src, dst, _ = after.reserve(new)
        assert same(again[0], after.table) and same(again[1], after.refs) and same(again[2], src)


@pytest.mark.parametrize("B,most", [(1, 9000), (3, 5000), (40, 700), (1000, 9)])
def test_reserve_many_pages_at_once(B, most):
    """Prompts: columns by the thousand, some of which have a page already."""
    rng = random.Random(B)
    page, columns = 16, 9003
    pages = B * most + 50
    order = list(range(pages))
    rng.shuffle(order)
    table, refs, length, new = [], [0] * pages, [], []
    for b in range(B):
        had, wants = rng.randint(0, 20), most if b % 3 == 0 else rng.randint(0, most)
        n = min(had, wants)
        row = [order.pop() for _ in range(n)] + [-1] * (columns - n)
        for i in range(n, wants):
            if rng.random() < 0.1:
                row[i] = order.pop()
        for e in row:
            if e >= 0:
                refs[e] += 1
        table.append(row)
        length.append(max(0, n * page - rng.randint(0, 15)) if n else 0)
        new.append(max(length[-1], wants * page - rng.randint(0, 15)))
    for spare in (0, 1):
        book = Book(table, refs, length, page)
        if spare:                  # one page too few
            free = [p for p, r in enumerate(refs) if r == 0]
            needed = sum(row[i] == -1 for row, n in zip(table, new) for i in range(-(-n // page)))
            for p in free[:len(free) - needed + 1]:
                book.refs[p] = 1
        want = book.copy()
        src, dst, missing = want.reserve(new)
        assert missing == spare
        ws = workspace(pages)
        got = sa.pages_reserve(*on_device(book), ints(new), page, workspace=ws)
        assert sa.read_status(ws) == (sa.E_OUT_OF_PAGES if spare else sa.OK) and int(ws.view(torch.int32)[1]) == missing
        assert same(got[0], want.table) and same(got[1], want.refs) and same(got[2], src) and same(got[3], dst)


def test_too_few_pages_goes_before_other_reports():
    book = Book([[0, -1, -1], [1, -1, -1], [2, -1, -1]], [1, 1, 1, 0], [16, 16, 10], 16)
    ws = workspace(4)
    got = sa.pages_reserve(*on_device(book), ints([48, 15, 10]), 16, workspace=ws)           # two pages; fewer tokens than there are
    assert sa.read_status(ws) == sa.E_OUT_OF_PAGES and int(ws.view(torch.int32)[1]) == 1
    assert same(got[0], book.table) and same(got[1], book.refs)


def test_a_partly_filled_page_that_nobody_holds_is_reported():
    book = Book([[0, -1], [1, -1]], [1, 0, 0], [10, 10], 16)
    ws = workspace(3)
    sa.pages_reserve(*on_device(book), ints([12, 12]), 16, workspace=ws)
    assert sa.read_status(ws) == sa.E_BAD_INDEX


def test_reserve_to_the_last_page():
    for spare in (0, 1, 2, 3, 4, 5):
        book = Book([[0, 1, -1, -1], [0, 1, -1, -1], [5, -1, -1, -1]], [2, 2, 0, 0, 0, 1] + [0] * spare, [24, 24, 16], 16)
        new = [40, 30, 50]        # a copy and a page; the first keeps what both go on in; three pages
        want = book.copy()
        src, dst, missing = want.reserve(new)
        assert (missing > 0) == (spare < 2)
        ws = workspace(6 + spare)
        got = sa.pages_reserve(*on_device(book), ints(new), 16, workspace=ws)
        assert sa.read_status(ws) == (sa.E_OUT_OF_PAGES if missing else sa.OK) and int(ws.view(torch.int32)[1]) == missing
        assert same(got[0], want.table) and same(got[1], want.refs) and same(got[2], src) and same(got[3], dst)


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "-".join(str(x) for x in s))
@pytest.mark.parametrize("rule", [(1, 0, 0), (1, 50, 4), (1, 1, 0), (40, 2, 40), (1560, 3, 1560), (7, 20, 1000000)])
def test_trim(size, rule):
    rng = random.Random(sum(rule))
    book = make_book(rng, *size)
    if rule[1] == 0:      # drafted tokens that were not taken
        book.len = [max(0, n - rng.choice((0, 1, 5, 100, n))) for n in book.len]
    want = book.copy()
    want.trim(*rule)
    table, length, refs = on_device(book)
    ws = workspace(size[1])
    args = dict(frame_tokens=rule[0], window=rule[1], sink=rule[2], workspace=ws)
    got = sa.pages_trim(table, length, refs, size[2], **args)
    assert sa.read_status(ws) == sa.OK
    assert same(got[0], want.table) and same(got[1], want.refs)
    assert same(table, book.table) and same(refs, book.refs)
    sa.pages_trim(table, length, refs, size[2], page_table_out=table, refs_out=refs, **args)
    assert sa.read_status(ws) == sa.OK and same(table, want.table) and same(refs, want.refs)
    sa.pages_trim(table, length, refs, size[2], page_table_out=table, refs_out=refs, **args)
    assert sa.read_status(ws) == sa.OK and same(table, want.table) and same(refs, want.refs)      # nothing is left to give back


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "-".join(str(x) for x in s))
@pytest.mark.parametrize("gone", [0.0, 0.5, 0.97, 1.0])
def test_compact(size, gone):
    rng = random.Random(int(gone * 10))
    book = make_book(rng, *size)
    parent = [-1 if rng.random() < gone else b for b in range(size[0])]
    book.fork(parent)
    want = book.copy()
    src, dst = want.compact()
    table, _, refs = on_device(book)
    ws = workspace(size[1])
    got = sa.pages_compact(table, refs, workspace=ws)
    assert sa.read_status(ws) == sa.OK
    assert same(got[0], want.table) and same(got[1], want.refs) and same(got[2], src) and same(got[3], dst)
    assert same(table, book.table) and same(refs, book.refs)
    sa.pages_compact(table, refs, page_table_out=table, refs_out=refs, workspace=ws)
    assert sa.read_status(ws) == sa.OK and same(table, want.table) and same(refs, want.refs)
    again = sa.pages_compact(table, refs, check_status=True)
    assert same(again[0], want.table) and (again[2] == -1).all()


def test_numbers_that_make_no_sense_are_reported():
    """Each is reported, nothing outside the book is touched, and the rest of the call is as without it."""
    table = [[0, 1, -1], [2, 3, 4], [5, -1, -1]]
    refs, length, P = [1] * 6 + [0] * 10, [30, 40, 10], 16

    def status(call):
        ws = workspace(16)
        got = call(ws)
        return sa.read_status(ws), got

    book = Book(table, refs, length, P)
    for parent in ([3, 1, 2], [0, -2, 2]):
        code, got = status(lambda ws: sa.pages_fork(*on_device(book), ints(parent), workspace=ws))
        want = book.copy()
        want.fork(parent)
        assert code == sa.E_BAD_INDEX and same(got[0], want.table) and same(got[1], want.len) and same(got[2], want.refs)
    for b, i, e in ((0, 1, 16), (1, 2, -5)):
        bad = book.copy()
        bad.table[b][i] = e
        code, got = status(lambda ws: sa.pages_fork(*on_device(bad), ints([2, 2, 2]), workspace=ws))
        want = bad.copy()
        want.fork([2, 2, 2])
        assert code == sa.E_BAD_INDEX and same(got[0], want.table) and same(got[2], want.refs)
    low = book.copy()
    low.refs[3] = 0
    assert status(lambda ws: sa.pages_fork(*on_device(low), ints([0, 0, 2]), workspace=ws))[0] == sa.E_BAD_INDEX
    for new in ([29, 48, 20], [49, 48, 20]):         # less than there is; more than the table holds
        code, got = status(lambda ws: sa.pages_reserve(*on_device(book), ints(new), P, workspace=ws))
        want = book.copy()
        src, dst, _ = want.reserve(new)
        assert code == sa.E_BAD_INDEX and same(got[0], want.table) and same(got[1], want.refs) and same(got[2], src)
    bad = book.copy()
    bad.len = [30, 40, -1]
    assert status(lambda ws: sa.pages_reserve(*on_device(bad), ints([31, 41, 20]), P, workspace=ws))[0] == sa.E_BAD_INDEX
    bad = book.copy()
    bad.table[0][1] = 99                                # the partly filled page
    assert status(lambda ws: sa.pages_reserve(*on_device(bad), ints([33, 40, 10]), P, workspace=ws))[0] == sa.E_BAD_INDEX
    for n in (-1, 49):
        bad = book.copy()
        bad.len[1] = n
        code, got = status(lambda ws: sa.pages_trim(*on_device(bad), P, window=5, workspace=ws))
        want = bad.copy()
        want.trim(1, 5, 0)
        assert code == sa.E_BAD_INDEX and same(got[0], want.table) and same(got[1], want.refs)
    for e in (16, -3):
        bad = book.copy()
        bad.table[1][0] = e
        code, got = status(lambda ws: sa.pages_trim(*on_device(bad), P, window=5, workspace=ws))
        want = bad.copy()
        want.trim(1, 5, 0)
        assert code == sa.E_BAD_INDEX and same(got[0], want.table) and same(got[1], want.refs)
    low = book.copy()
    low.refs[2] = 0
    assert status(lambda ws: sa.pages_trim(*on_device(low), P, window=5, workspace=ws))[0] == sa.E_BAD_INDEX
    for e in (16, -3, 9):                               # 9: nobody holds it
        bad = book.copy()
        bad.table[1][0] = e
        code, got = status(lambda ws: sa.pages_compact(ints(bad.table), ints(bad.refs), workspace=ws))
        want = bad.copy()
        want.compact()
        assert code == sa.E_BAD_INDEX and same(got[0], want.table) and same(got[1], want.refs)


# ------------------------------------------------------------------------------------------------------------------ copy

def clone(cache):
    return sa.KVCache(*(None if x is None else x.clone(memory_format=torch.preserve_format) for x in cache))


COPIES = [
    # pages, H, page, d, fp8, layout, pairs
    (5, 1, 16, 64, True, "hnd", 1),
    (9, 3, 16, 64, False, "nhd", 3),
    (300, 8, 16, 128, True, "hnd", 150),
    (300, 7, 128, 128, False, "nhd", 100),
    (40, 12, 128, 128, True, "nhd", 17),
    (40, 5, 32, 64, True, "padded", 20),
    (3000, 1, 16, 64, False, "padded", 1500),
]


def pool(gen, pages, H, page, d, fp8, layout):
    if layout != "padded":
        return make_cache(gen, pages, H, page, d, fp8, layout=layout)
    cache = make_cache(gen, pages, H + 1, page * 2, d, fp8)          # heads and tokens of a larger pool
    part = [x[:, 1:, :page] for x in cache[:2]]
    return sa.KVCache(*part, *(None if s is None else s[:, 1:].contiguous() for s in cache[2:]))


@pytest.mark.parametrize("case", COPIES, ids=lambda c: "-".join(str(x) for x in c))
def test_copy(case):
    pages, H, page, d, fp8, layout, n = case
    gen = torch.Generator(device=DEV).manual_seed(pages + H)
    rng = random.Random(n)
    cache = pool(gen, pages, H, page, d, fp8, layout)
    chosen = rng.sample(range(pages), min(2 * n, pages))
    dst, rest = chosen[:n], chosen[n:] or [p for p in range(pages) if p not in chosen[:n]]
    src = [rng.choice(rest) for _ in dst]
    pairs = [(a, b) for a, b in zip(src, dst)] + [(-1, -1)] * (n // 2)
    rng.shuffle(pairs)
    src, dst = (list(x) for x in zip(*pairs))
    keep = [(a, b) for a, b in pairs if a >= 0]

    def expect(to, by):
        want = clone(to)
        for x, y in zip(want, by):
            if x is not None:
                bits = (lambda t: t.view(torch.uint8)) if x.element_size() == 1 else (lambda t: t)
                bits(x)[ints([b for _, b in keep]).long()] = bits(y)[ints([a for a, _ in keep]).long()]
        return want

    for other in (None, "hnd", "nhd", "padded"):
        to = cache if other is None else pool(gen, pages + 4, H, page, d, fp8, other)
        want = expect(to, clone(cache))
        ws = torch.full((256,), 0xA5, dtype=torch.uint8, device=DEV)
        before = clone(cache)
        sa.cache_copy_pages(cache, ints(src), ints(dst), to=None if other is None else to, workspace=ws)
        assert sa.read_status(ws) == sa.OK
        for got, ref in zip(to, want):
            assert (got is None) == (ref is None) and (got is None or same_bits(got, ref))
        if other is None:
            cache = to
        else:
            assert all(x is None or same_bits(x, y) for x, y in zip(cache, before))


def test_copy_leaves_what_lies_between_the_pages():
    gen = torch.Generator(device=DEV).manual_seed(6)
    big = make_cache(gen, 6, 4, 64, 128, True)
    part = sa.KVCache(big.k[:, 1:3, 16:32], big.v[:, 1:3, 16:32], big.k_scale[:, 1:3].contiguous(), big.v_scale[:, 1:3].contiguous())
    before = clone(big)
    sa.cache_copy_pages(part, ints([0, 4]), ints([3, 1]), check_status=True)
    for x, y in zip(big[:2], before[:2]):
        want = y.view(torch.uint8).clone()
        for a, b in ((0, 3), (4, 1)):
            want[b, 1:3, 16:32] = y.view(torch.uint8)[a, 1:3, 16:32]
        assert torch.equal(x.view(torch.uint8), want)


@pytest.mark.parametrize("word", [0, -7, 0x5A5A5A5A])
@pytest.mark.parametrize("pages", [50, 300000])
def test_copy_reports(word, pages):
    """Pairs that name no page are passed over; a page that is written twice, or written and read, is reported."""
    cache = sa.alloc_cache(pages, 1, 16, 64, fp8=False, device=DEV)
    cache.k.copy_(torch.arange(pages, device=DEV).remainder(251)[:, None, None, None].expand_as(cache.k))
    top = pages - 1
    other = sa.alloc_cache(20, 1, 16, 64, fp8=False, device=DEV)
    ws = torch.zeros(64, dtype=torch.int32, device=DEV)
    for src, dst, to, code in (([1, 2, top], [3, 4, 5], None, sa.OK), ([1, 1, -1], [top, 4, -1], None, sa.OK), ([1, 2], [pages, 4], None, sa.E_BAD_INDEX),
                               ([-1, 2], [3, 4], None, sa.E_BAD_INDEX), ([pages, 2], [3, 4], None, sa.E_BAD_INDEX), ([1, 2], [-7, 4], None, sa.E_BAD_INDEX),
                               ([1, 2], [9, 9], None, sa.E_BAD_INDEX), ([1, top - 1], [top - 1, 9], None, sa.E_BAD_INDEX), ([8, 2], [8, 9], None, sa.E_BAD_INDEX),
                               ([8, 2], [8, 2], other, sa.OK), ([8, 2], [8, 8], other, sa.E_BAD_INDEX), ([8, 2], [8, 20], other, sa.E_BAD_INDEX),
                               ([8] * 5000 + [2], [-1] * 5000 + [9], None, sa.E_BAD_INDEX), ([-1] * 5000, [-1] * 5000, None, sa.OK)):
        ws[0] = word
        before = cache.k.clone()
        sa.cache_copy_pages(cache, ints(src), ints(dst), to=to, workspace=ws.view(torch.uint8))
        assert sa.read_status(ws.view(torch.uint8)) == code, (src[:3], dst[:3])
        if to is None:
            want = before.clone()
            if len(set(dst)) == len(dst) and not set(src) & set(dst):
                for a, b in zip(src, dst):
                    if 0 <= a < pages and 0 <= b < pages:
                        want[b] = before[a]
                assert torch.equal(cache.k, want)
            cache.k.copy_(before)
    empty = torch.empty(0, dtype=torch.int32, device=DEV)
    ws[0] = word
    sa.cache_copy_pages(cache, empty, empty, workspace=ws.view(torch.uint8))
    assert sa.read_status(ws.view(torch.uint8)) == sa.OK


def test_captured_with_counts_that_change():
    """One graph of reserve, copy and trim in place, replayed step after step, against the lists."""
    rng = random.Random(4)
    P, B, columns, pages = 16, 6, 30, 140
    book = make_book(rng, B, pages, P, columns, 60, share=0.8, pinned=0.0)
    table, length, refs = on_device(book)
    new = length.clone()
    cache = make_cache(torch.Generator(device=DEV).manual_seed(1), pages, 2, P, 64, True)
    src, dst = torch.empty_like(length), torch.empty_like(length)
    ws = [workspace(pages) for _ in range(3)]

    def step():
        sa.pages_reserve(table, length, refs, new, P, page_table_out=table, refs_out=refs, src=src, dst=dst, workspace=ws[0])
        sa.cache_copy_pages(cache, src, dst, workspace=ws[1])
        length.copy_(new)
        sa.pages_trim(table, length, refs, P, window=50, sink=20, page_table_out=table, refs_out=refs, workspace=ws[2])

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    table.copy_(ints(book.table)); length.copy_(ints(book.len)); refs.copy_(ints(book.refs))
    for _ in range(12):
        more = [min(n + rng.choice((0, 1, 7, 33)), columns * P) for n in book.len]
        new.copy_(ints(more))
        held = cache.k.view(torch.uint8).clone()
        graph.replay()
        want_src, want_dst, missing = book.reserve(more)
        assert not missing and same(src, want_src) and same(dst, want_dst)
        book.len = more
        book.trim(1, 50, 20)
        assert [sa.read_status(w) for w in ws] == [sa.OK] * 3
        assert same(table, book.table) and same(refs, book.refs)
        for a, b in zip(want_src, want_dst):
            if a >= 0:
                held[b] = held[a]
        assert torch.equal(cache.k.view(torch.uint8), held)


def test_copy_far_apart():
    """Pages whose places lie more than 2^32 bytes apart."""
    pages, H = 36000, 8
    cache = sa.KVCache(*(torch.zeros((pages, H, 64, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2)))
    assert cache.k[0].numel() * 2 * pages > 2 ** 32
    gen = torch.Generator(device=DEV).manual_seed(1)
    far = (0, 1, pages // 2, pages - 2, pages - 1)
    for p in far:
        cache.k[p], cache.v[p] = (torch.randn((H, 64, 128), generator=gen, device=DEV).bfloat16() for _ in range(2))
    want = {b: (cache.k[a].clone(), cache.v[a].clone()) for a, b in ((0, pages - 3), (pages - 1, 2), (pages - 2, 3), (pages // 2, pages - 4))}
    src, dst = ints([0, pages - 1, pages - 2, pages // 2]), ints(list(want))
    sa.cache_copy_pages(cache, src, dst, check_status=True)
    for b, (k, v) in want.items():
        assert same_bits(cache.k[b], k) and same_bits(cache.v[b], v)
