"""Reservation of pages where sequences were forked behind pages reserved ahead, or taken back behind pages that others hold: the book against
the same steps taken entry after entry, and sequences that go on apart over one pool."""
import random

import pytest
import torch

import paper_2609_23153_b200 as sa
from test_gpu_cache import DEV, same_bits
from test_gpu_pages import SIZES, Book, ints, make_book, on_device, same, workspace

pytestmark = pytest.mark.gpu


class Ahead(Book):
    """A reservation in which a column behind the length keeps its page only if nobody else holds it."""

    def reserve(self, new):
        P, held = self.page, list(self.refs)
        free = [p for p, r in enumerate(held) if r == 0]
        active = [0 <= n <= m <= len(self.table[0]) * P and m > n for n, m in zip(self.len, new)]
        writers = {}
        for b, n in enumerate(self.len):
            if active[b] and n % P:
                e = self.table[b][n // P]
                if self.there(e) and held[e] > 1:
                    writers.setdefault(e, []).append(b)
        copies = {b for e, w in writers.items() for b in (w if len(w) != held[e] else w[1:])}
        wanted = []
        for b, n in enumerate(self.len):
            if active[b]:
                wanted += [(b, n // P)] if b in copies else []
                wanted += [(b, i) for i in range(-(-n // P), -(-new[b] // P)) if self.table[b][i] == -1 or self.there(self.table[b][i]) and held[self.table[b][i]] > 1]
        src, dst = [-1] * len(new), [-1] * len(new)
        if len(wanted) > len(free):
            return src, dst, len(wanted) - len(free)
        for (b, i), p in zip(wanted, free):
            e = self.table[b][i]
            if i < -(-self.len[b] // P):
                src[b], dst[b] = e, p
            if self.there(e):
                self.refs[e] -= 1
            self.table[b][i] = p
            self.refs[p] += 1
        return src, dst, 0


def ahead_book(rng, size, most_ahead):
    """Some sequences have pages ahead of their tokens, then all fork; some children go back a few tokens."""
    B, pages, page, columns, _ = size
    made = make_book(rng, *size)
    book = Ahead(made.table, made.refs, made.len, page)
    spare = [p for p, r in enumerate(book.refs) if r == 0]
    rng.shuffle(spare)
    for b in range(B):
        first = -(-book.len[b] // page)
        for i in range(first, min(first + rng.randint(0, most_ahead), columns)):
            if len(spare) > pages // 4 and rng.random() < 0.9:
                book.table[b][i] = spare.pop()
                book.refs[book.table[b][i]] = 1
    book.fork([rng.choice((b, b, rng.randrange(B))) for b in range(B)])
    book.len = [max(0, n - rng.choice((0, 0, 1, page, rng.randint(0, 3 * page)))) for n in book.len]
    return book


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "-".join(str(x) for x in s))
@pytest.mark.parametrize("seed", range(4))
def test_pages_ahead_that_others_hold(size, seed):
    rng = random.Random(200 + seed)
    B, pages, page, columns, most = size
    book = ahead_book(rng, size, (1, 3, 8, 300)[seed])
    step = (1, page // 2, 3 * page, 290 * page)[seed]
    new = [min(n + rng.choice((0, 1, step, rng.randint(0, step))), columns * page) for n in book.len]
    want = book.copy()
    want.__class__ = Ahead
    src, dst, missing = want.reserve(new)
    table, length, refs = on_device(book)
    ws = workspace(pages)
    got = sa.pages_reserve(table, length, refs, ints(new), page, workspace=ws)
    assert sa.read_status(ws) == (sa.E_OUT_OF_PAGES if missing else sa.OK) and int(ws.view(torch.int32)[1]) == missing
    assert same(got[0], want.table) and same(got[1], want.refs) and same(got[2], src) and same(got[3], dst)
    assert same(table, book.table) and same(refs, book.refs)
    sa.pages_reserve(table, length, refs, ints(new), page, page_table_out=table, refs_out=refs, workspace=ws)
    assert same(table, want.table) and same(refs, want.refs)
    if not missing:
        # counts are the entries' and the other holders', as before, and new tokens lie in pages of one holder
        others = [r.cpu() - torch.bincount(t[t >= 0].cpu().long(), minlength=pages) for t, r in ((ints(book.table), ints(book.refs)), (table, refs))]
        assert torch.equal(*others)
        pages_of_new = [table[b, n // page:-(-m // page)] for b, (n, m) in enumerate(zip(book.len, new)) if m > n]
        if pages_of_new:
            assert (refs[torch.cat(pages_of_new).long()] == 1).all()


@pytest.mark.parametrize("length,new,columns", [(64, 65, {4}), (60, 70, {3, 4}), (64, 96, {4, 5}), (70, 80, {4})])
def test_two_children_of_one_that_had_pages_ahead(length, new, columns):
    """Pages of 16, six reserved, forked from one another: every column that both go on in has two pages."""
    book = Book([list(range(6)), [-1] * 6], [1] * 6 + [0] * 10, [length, 0], 16)
    book.fork([0, 0])
    assert book.refs[:6] == [2] * 6
    ws = workspace(16)
    table, refs, src, dst = sa.pages_reserve(*on_device(book), ints([new, new]), 16, workspace=ws)
    assert sa.read_status(ws) == sa.OK
    apart = {i for i in range(6) if int(table[0, i]) != int(table[1, i])}
    assert apart == columns
    held = torch.bincount(table.flatten().long(), minlength=16).int()
    assert torch.equal(refs, held)
    # the first keeps the partly filled one, the second copies it; what lies behind has nothing to copy
    assert src.tolist() == ([-1, -1] if length % 16 == 0 else [-1, length // 16]) and dst.tolist()[0] == -1


def test_pages_ahead_that_somebody_else_keeps():
    book = Ahead([[0, 1, 2, -1]], [1, 2, 1, 0, 0, 0], [16], 16)
    want = Ahead(book.table, book.refs, book.len, 16)
    want.reserve([60])
    table, refs, src, dst = sa.pages_reserve(*on_device(book), ints([60]), 16, check_status=True)
    assert table.tolist() == want.table == [[0, 3, 2, 4]] and refs.tolist() == want.refs == [1, 1, 1, 1, 1, 0] and src.tolist() == dst.tolist() == [-1]


def test_too_few_pages_for_those_that_others_hold():
    """All or nothing: nobody's page is taken and no count falls."""
    book = Ahead([[0, 1, 2], [0, 1, 2], [3, -1, -1]], [2, 2, 2, 1] + [0] * 3, [16, 16, 16], 16)
    ws = workspace(7)
    got = sa.pages_reserve(*on_device(book), ints([48, 33, 16]), 16, workspace=ws)          # two of the first, two of the second
    assert sa.read_status(ws) == sa.E_OUT_OF_PAGES and int(ws.view(torch.int32)[1]) == 1
    assert same(got[0], book.table) and same(got[1], book.refs) and (got[2] == -1).all() and (got[3] == -1).all()


def gathered(x, row, n, page):
    """Bytes of a sequence's first n tokens."""
    at = torch.arange(n, device=DEV)
    y = x[row[at // page].long(), :, at % page]
    return y.view(torch.uint8) if y.element_size() == 1 else y


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("length,ahead,more", [(64, 32, 1), (60, 40, 30), (17, 100, 90), (0, 50, 20)])
def test_forked_behind_pages_ahead_go_on_apart(fp8, length, ahead, more):
    """Reserved ahead, some of it taken, forked without a trim, reserved, appended: each of the three has the tokens that it would have alone."""
    P, H, d, pages, columns = 16, 2, 64, 80, 16
    gen = torch.Generator(device=DEV).manual_seed(length + more)
    rows = lambda n: torch.randn((n, H, d), generator=gen, device=DEV).bfloat16()
    table, refs = torch.full((1, columns), -1, dtype=torch.int32, device=DEV), torch.zeros(pages, dtype=torch.int32, device=DEV)
    cache = sa.alloc_cache(pages, H, P, d, fp8=fp8, device=DEV)
    table, refs, _, _ = sa.pages_reserve(table, ints([0]), refs, ints([length + ahead]), P, check_status=True)
    first = [rows(length) for _ in range(2)]
    if length:
        sa.cache_append(cache, *first, table, ints([length]), check_status=True)
    table, lens, refs = sa.pages_fork(table, ints([length]), refs, ints([0, 0, 0]), check_status=True)
    counts = [more, more // 2 + 1, more]
    kv_len = ints([length + c for c in counts])
    table, refs, src, dst = sa.pages_reserve(table, lens, refs, kv_len, P, check_status=True)
    for i in range(length // P, -(-(length + max(counts)) // P)):
        mine = [int(table[b, i]) for b in range(3) if i * P < length + counts[b]]
        assert len(set(mine)) == len(mine)                                        # (else the appending below would be a race)
    sa.cache_copy_pages(cache, src, dst, check_status=True)
    new = [[rows(c) for _ in range(2)] for c in counts]
    q_start = ints([0, counts[0], counts[0] + counts[1], sum(counts)])
    batch = dict(q_start=q_start, max_new=max(counts), check_status=True)
    sa.cache_append(cache, *(torch.cat([n[i] for n in new]) for i in range(2)), table, kv_len, **batch)
    q = torch.randn((sum(counts), 4, d), generator=gen, device=DEV).bfloat16()
    out = sa.cache_fwd(q, cache, table, kv_len, **batch)
    for b, c in enumerate(counts):
        n = length + c
        alone = sa.alloc_cache(columns, H, P, d, fp8=fp8, device=DEV)
        own = torch.arange(columns, dtype=torch.int32, device=DEV)[None].contiguous()
        if length:
            sa.cache_append(alone, *first, own, ints([length]))
        sa.cache_append(alone, *new[b], own, ints([n]), max_new=c, q_start=ints([0, c]))
        for x, y in zip(cache[:2], alone[:2]):
            assert torch.equal(gathered(x, table[b], n, P), gathered(y, own[0], n, P))
        # both attentions round their weights and their output to bf16, by half a step of 2^-8 at most each
        at = slice(int(q_start[b]), int(q_start[b + 1]))
        want = sa.cache_fwd(q[at].contiguous(), alone, own, ints([n]), max_new=c, q_start=ints([0, c])).double()
        assert ((out[at].double() - want).abs() <= 2.0 ** -7 * (want.abs() + max(float(first[1].abs().max()) if length else 0.0, float(new[b][1].abs().max())))).all()


def test_a_sequence_taken_back_leaves_what_others_go_on_in():
    """One of two goes back behind a page that the other writes to: neither touches the other's tokens."""
    P, H, d = 16, 1, 64
    gen = torch.Generator(device=DEV).manual_seed(3)
    cache = sa.alloc_cache(12, H, P, d, fp8=False, device=DEV)
    book = Book([[0, 1, 2, -1], [0, 1, 2, -1]], [2, 2, 2] + [0] * 9, [40, 20], P)          # page 2 holds tokens 32 to 39 of the first; the second is back at 20
    table, length, refs = on_device(book)
    k, v = (torch.randn((40, H, d), generator=gen, device=DEV).bfloat16() for _ in range(2))
    sa.cache_append(cache, k, v, table[:1].contiguous(), ints([40]), check_status=True)
    new = ints([41, 45])
    table, refs, src, dst = sa.pages_reserve(table, length, refs, new, P, check_status=True)
    assert int(table[0, 2]) != int(table[1, 2]) and int(table[0, 1]) != int(table[1, 1])
    sa.cache_copy_pages(cache, src, dst, check_status=True)
    more = [torch.randn((26, H, d), generator=gen, device=DEV).bfloat16() for _ in range(2)]
    sa.cache_append(cache, *more, table, new, q_start=ints([0, 1, 26]), max_new=25, check_status=True)
    for x, y, z in zip(cache[:2], (k, v), more):
        assert torch.equal(gathered(x, table[0], 41, P), torch.cat([y, z[:1]]))
        assert torch.equal(gathered(x, table[1], 45, P), torch.cat([y[:20], z[1:]]))


@pytest.mark.parametrize("columns", [4, 500])
def test_entries_that_name_no_page_count_as_none(columns):
    """-1 or any other number outside the pool, in a column that is asked for."""
    pages, P = 2 * columns + 10, 16
    wrong = [-1, -2, pages, 2 ** 31 - 1, -2 ** 31, pages + 7, -1]
    row = [0, 1] + [wrong[i % len(wrong)] for i in range(columns - 2)]
    table, refs = [row, [2, -2] + row[2:]], [1, 1, 1] + [0] * (pages - 3)
    length, new = [20, 16], [columns * P, (columns - 1) * P]
    got = sa.pages_reserve(ints(table), ints(length), ints(refs), ints(new), P, check_status=True)
    first = list(range(3, 3 + columns - 2))
    second = list(range(3 + columns - 2, 3 + 2 * columns - 4))
    assert got[0].tolist() == [[0, 1] + first, [2] + second + [row[-1]]]
    assert got[1].tolist() == [1] * (3 + 2 * columns - 4) + [0] * (pages - 3 - 2 * columns + 4)
    assert (got[2] == -1).all() and (got[3] == -1).all()
    few = [1] * pages                                  # none is free: the book stays as it was
    ws = workspace(pages)
    got = sa.pages_reserve(ints(table), ints(length), ints(few), ints(new), P, workspace=ws)
    assert sa.read_status(ws) == sa.E_OUT_OF_PAGES and int(ws.view(torch.int32)[1]) == 2 * columns - 4
    assert same(got[0], table) and same(got[1], few)


@pytest.mark.parametrize("columns,at", [(4, 2), (4, 3), (500, 2), (500, 499)])
def test_a_page_ahead_that_nobody_holds_is_reported(columns, at):
    """It stays where it is, and the rest of the call is as without it."""
    pages, P = 2 * columns, 16
    row = [0] + [-1] * (columns - 1)
    row[at] = pages - 1
    ws = workspace(pages)
    got = sa.pages_reserve(ints([row]), ints([16]), ints([1] + [0] * (pages - 1)), ints([columns * P]), P, workspace=ws)
    assert sa.read_status(ws) == sa.E_BAD_INDEX and int(ws.view(torch.int32)[1]) == pages - 1
    free = iter(range(1, pages))
    assert got[0].tolist() == [[e if e >= 0 else next(free) for e in row]]
    sa.pages_reserve(ints([row]), ints([16]), ints([1] + [0] * (pages - 1)), ints([at * P]), P, workspace=ws)      # not asked for: not looked at
    assert sa.read_status(ws) == sa.OK


def lengths_of_the_step(book, new, missing):
    """... of a book whose numbers make sense."""
    return [m if m == n or not missing else -1 for n, m in zip(book.len, new)]


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "-".join(str(x) for x in s))
@pytest.mark.parametrize("seed", range(3))
def test_lengths_for_the_step(size, seed):
    rng = random.Random(300 + seed)
    B, pages, page, columns, most = size
    book = ahead_book(rng, size, 3)
    new = [min(n + rng.choice((0, 1, page, 40 * page)[:seed + 2]), columns * page) for n in book.len]
    if seed == 1:
        book.refs = [max(r, 1) for r in book.refs]        # none is free
    want = book.copy()
    want.__class__ = Ahead
    src, dst, missing = want.reserve(new)
    for in_place in (False, True):
        table, length, refs = on_device(book)
        kv_len = torch.full((B,), 77, dtype=torch.int32, device=DEV)
        there = dict(page_table_out=table, refs_out=refs) if in_place else {}
        got = sa.pages_reserve(table, length, refs, ints(new), page, kv_len_out=kv_len, **there)
        assert same(got[0], want.table) and same(got[1], want.refs) and same(got[2], src) and same(got[3], dst)
        assert same(kv_len, lengths_of_the_step(book, new, missing))


@pytest.mark.parametrize("columns", [5, 300])
def test_a_sequence_that_has_not_got_its_pages_has_no_length(columns):
    """By its own numbers, each in another way; the others have theirs."""
    P, far = 16, 16 * columns
    table = [[0] + [-1] * (columns - 1), [1] + [-1] * (columns - 1), [-1] * columns, [3] + [-1] * (columns - 1), [4, columns + 60] + [-1] * (columns - 2), [5] + [-1] * (columns - 1)]
    refs = [1, 1, 0, 0, 1, 1] + [0] * (6 * columns + 200)
    length, new = [16, 16, 10, 10, 16, 16], [far, 15, 12, 12, far, far + 1]
    kv_len = ints([77] * 6)
    ws = workspace(len(refs))
    got = sa.pages_reserve(ints(table), ints(length), ints(refs), ints(new), P, kv_len_out=kv_len, workspace=ws)
    assert sa.read_status(ws) == sa.E_BAD_INDEX
    # fewer than there are; a partly filled page that is none, or nobody's; a page ahead that is nobody's; more than the table holds
    assert kv_len.tolist() == [far, -1, -1, -1, -1, -1] and (got[0][0] >= 0).all()


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("new,G", [(1, 2), (5, 4), (40, 8)])
def test_captured_step_whose_pages_do_not_suffice(fp8, new, G):
    """Reserve, copy, append, attend and trim in one graph.  Two sequences share a partly filled page and the pool runs out: nothing that a page
    holds changes, and the book stays; with pages given back the same graph goes on."""
    P, H, d, B, columns = 16, 2, 64, 3, 12
    need = -(-(20 + new) // P) - 2                        # further pages of each
    pages = 2 + 4 + 2 * need                              # two shared, four of the third, and one too few for a copy and what is new
    gen = torch.Generator(device=DEV).manual_seed(new)
    cache = sa.alloc_cache(pages, H, P, d, fp8=fp8, device=DEV)
    for x in cache:
        if x is not None:
            x.zero_() if x.element_size() != 4 else x.fill_(1.0)
    rows = lambda n, h: torch.randn((n, h, d), generator=gen, device=DEV).bfloat16()
    table, refs, lens = torch.full((2, columns), -1, dtype=torch.int32, device=DEV), torch.zeros(pages, dtype=torch.int32, device=DEV), ints([20, 64])
    table, refs, _, _ = sa.pages_reserve(table, ints([0, 0]), refs, lens, P, check_status=True)
    sa.cache_append(cache, rows(84, H), rows(84, H), table, lens, q_start=ints([0, 20, 84]), max_new=64, check_status=True)
    table, lens, refs = sa.pages_fork(table, lens, refs, ints([0, 0, 1]), check_status=True)
    want_new, kv_len, q_start = ints([20 + new, 20 + new, 64]), torch.empty_like(lens), ints([0, new, 2 * new, 2 * new])
    src, dst = torch.empty_like(lens), torch.empty_like(lens)
    k, v, q = rows(2 * new, H), rows(2 * new, H), rows(2 * new, H * G)
    turned, out = torch.empty_like(q), torch.empty_like(q)
    batch = dict(q_start=q_start, max_new=new)
    ws = [torch.zeros(1 << 12, dtype=torch.uint8, device=DEV) for _ in range(4)] + [torch.zeros(1 << 28, dtype=torch.uint8, device=DEV)]

    def step():
        sa.pages_reserve(table, lens, refs, want_new, P, page_table_out=table, refs_out=refs, src=src, dst=dst, kv_len_out=kv_len, workspace=ws[0])
        sa.cache_copy_pages(cache, src, dst, workspace=ws[1])
        turned.copy_(q)
        sa.cache_append(cache, k, v, table, kv_len, q=turned, q_out=turned, workspace=ws[2], **batch)
        sa.cache_fwd(turned, cache, table, kv_len, out=out, workspace=ws[4], **batch)
        sa.pages_trim(table, kv_len, refs, P, page_table_out=table, refs_out=refs, workspace=ws[3])

    before = [x.clone() for x in (table, refs)] + [x.clone() for x in cache if x is not None]

    def unchanged():
        now = [table, refs] + [x for x in cache if x is not None]
        return all(same_bits(x, y) for x, y in zip(now, before))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(2):
        graph.replay()
        assert [sa.read_status(w) for w in ws] == [sa.E_OUT_OF_PAGES, sa.OK, sa.E_BAD_INDEX, sa.E_BAD_INDEX, sa.E_BAD_INDEX]
        assert kv_len.tolist() == [-1, -1, 64] and unchanged() and (out == 0).all()
    # the third ends: there is room
    t, _, r = sa.pages_fork(table, lens, refs, ints([0, 1, -1]), check_status=True)
    table.copy_(t), refs.copy_(r), lens.copy_(ints([20, 20, 0])), want_new.copy_(ints([20 + new, 20 + new, 0]))
    graph.replay()
    assert [sa.read_status(w) for w in ws] == [sa.OK] * 5 and kv_len.tolist() == [20 + new, 20 + new, 0]
    for x, y, s in ((cache.k, k, cache.k_scale), (cache.v, v, cache.v_scale)):
        for b in range(2):
            at = torch.arange(20, 20 + new, device=DEV)
            pg = table[b][at // P].long()
            got = x.view(torch.uint8)[pg, :, at % P].view(torch.float8_e4m3fn).double() * s[pg].double()[..., None] if fp8 else x[pg, :, at % P].double()
            mine = y[b * new:(b + 1) * new].double()
            # a code is off by half a step, 2^-4 of it, or 2^-10 scales among the smallest
            assert ((got - mine).abs() <= (2.0 ** -4 * mine.abs() + (s[pg].double()[..., None] * 2.0 ** -10) if fp8 else torch.zeros_like(mine))).all()
    assert (out != 0).any(-1).all()
