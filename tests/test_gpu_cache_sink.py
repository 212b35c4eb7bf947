"""GPU parity of the attention over a paged cache through a window and with the first tokens, against softmax attention in 64 bits over
exactly the keys that a row sees.  Everything that no row sees holds NaN, and pages between the first tokens and the window are gone."""
import math

import pytest
import torch

import paper_2609_23153_b200 as sa
from test_gpu_cache import DEV, batch_of, check, make_cache, make_table, same_bits, visible

pytestmark = pytest.mark.gpu


def seen_keys(pos, length, frame, window, sink):
    lo, hi = visible(pos, length, frame, window)
    return [j for j in range(min(sink, lo, hi))] + list(range(lo, hi))


def reference(q, cache, table, lens, news, frame, window, sink):
    Hk, P, d = cache.k.shape[1:]
    T, H, _ = q.shape
    out = torch.zeros((T, H, d), dtype=torch.float64, device=DEV)
    lse = torch.full((T, H), -math.inf, dtype=torch.float64, device=DEV)
    t = 0
    for b, (length, n) in enumerate(zip(lens, news)):
        for i in range(n):
            keys = seen_keys(length - n + i, length, frame, window, sink)
            if keys:
                j = torch.tensor(keys, device=DEV)
                pg, slot = table[b, j // P].long(), j % P

                def rows(x, s):
                    y = x.view(torch.uint8)[pg, :, slot].view(torch.float8_e4m3fn).double() if s is not None else x[pg, :, slot].double()
                    return (y if s is None else y * s[pg].double()[..., None]).transpose(0, 1)
                a = torch.einsum("hgd,hjd->hgj", q[t].double().view(Hk, H // Hk, d), rows(cache.k, cache.k_scale)) * d ** -0.5
                lse[t] = torch.logsumexp(a, -1).view(H)
                out[t] = torch.einsum("hgj,hjd->hgd", torch.softmax(a, -1), rows(cache.v, cache.v_scale)).reshape(H, d)
            t += 1
    return out, lse


def hide(cache, table, lens, news, frame, window, sink):
    """(cache, table) with NaN and infinities in every token that no row sees, and no page where a page has none that is seen."""
    P, fp8 = cache.k.shape[2], cache.k_scale is not None
    owned = torch.zeros((cache.k.shape[0], P), dtype=torch.bool)
    table = table.clone()
    for b, (length, n) in enumerate(zip(lens, news)):
        seen = torch.zeros(table.shape[1] * P, dtype=torch.bool)
        for i in range(n):
            seen[seen_keys(length - n + i, length, frame, window, sink)] = True
        seen = seen.view(-1, P)
        for i in range(table.shape[1]):
            if seen[i].any():
                owned[int(table[b, i])] |= seen[i]
            else:
                table[b, i] = -1
    owned = owned.to(DEV)
    junk = torch.tensor([0x7f, 0xff, 0x7e, 0xfe] if fp8 else [0x7fc0, -0x0080, 0x7f80, 0x7f7f], device=DEV)
    pools = []
    for x in (cache.k, cache.v):
        bits = x.view(torch.uint8 if fp8 else torch.int16).clone(memory_format=torch.preserve_format)
        pattern = junk[torch.arange(bits.numel(), device=DEV) % 4].view(bits.shape).to(bits.dtype)
        pools.append(torch.where(owned[:, None, :, None], bits, pattern).view(x.dtype))
    scales = [None if s is None else torch.where(owned.any(1)[:, None], s, math.nan) for s in (cache.k_scale, cache.v_scale)]
    return sa.KVCache(*pools, *scales), table


CASES = [
    # lens, news, H, Hk, d, page, fp8, frame, window, sink
    ([1], [1], 8, 8, 128, 16, True, 1, 1, 1),
    ([2], [1], 8, 8, 128, 16, True, 1, 1, 1),
    ([500], [1], 8, 8, 64, 16, True, 1, 100, 4),
    ([1000, 1, 333, 128], [1, 1, 1, 1], 40, 8, 128, 64, True, 1, 100, 4),
    ([1000, 200, 333, 0], [1, 1, 1, 1], 12, 12, 64, 32, False, 1, 130, 33),
    ([2049, 7], [1, 1], 24, 2, 128, 32, False, 1, 17, 129),
    ([2049, 900], [1, 1], 24, 2, 128, 128, True, 1, 300, 127),
    ([900, 513], [3, 5], 16, 4, 128, 16, True, 1, 64, 16),
    ([900, 513], [3, 5], 16, 4, 64, 128, True, 1, 700, 130),            # first tokens and window in neighbouring tiles, or one
    ([600, 130], [1, 1], 4, 2, 128, 64, True, 1, 200, 5000),            # more first tokens than there are
    ([1500, 800], [1, 4], 6, 3, 128, 128, True, 50, 2, 50),
    ([40000, 300], [1, 1], 2, 2, 128, 64, True, 1, 9000, 777),
    ([40000, 41000], [2, 2], 4, 4, 64, 16, False, 1, 30000, 1),
    ([5000, 6000, 70], [1, 1, 1], 64, 4, 128, 64, True, 1, 64, 640),    # sixteen rows
    ([9000, 8], [33, 8], 40, 8, 128, 64, True, 1, 500, 4),
    ([2000, 1600, 40], [40, 90, 17], 2, 1, 64, 128, True, 1, 33, 200),
    ([7000], [40], 3, 1, 64, 64, False, 1, 128, 128),
    ([2000, 0, 515], [300, 4, 257], 8, 2, 128, 16, True, 1, 100, 20),
    ([1300, 900], [700, 300], 4, 4, 128, 128, True, 100, 3, 100),
    ([1300, 900], [700, 300], 5, 5, 128, 32, False, 1, 256, 300),
    ([1300, 400], [700, 300], 5, 5, 64, 32, True, 1, 20, 129),
    ([4000], [1000], 2, 2, 128, 64, False, 250, 2, 250),
    ([3, 130, 513], [7, 130, 1], 7, 7, 128, 64, True, 1, 50, 3),        # more new tokens than the first sequence holds
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) for x in c[2:]) + f"-{len(c[0])}x{max(c[0])}")
@pytest.mark.parametrize("spare", [1, 700])
def test_window_and_first_tokens(case, spare):
    """`spare`: columns of the table behind the sequences', which decide about cluster or line."""
    lens, news, H, Hk, d, page, fp8, frame, window, sink = case
    gen = torch.Generator(device=DEV).manual_seed(sum(lens) + H + sink)
    pages = sum(-(-n // page) for n in lens) + 2
    cache = make_cache(gen, pages, Hk, page, d, fp8, general=True, layout="nhd" if spare == 1 else "hnd")
    table = make_table(gen, lens, page, pages, spare)
    kv_len, q_start = batch_of(lens, news)
    q = (1.5 * torch.randn((sum(news), H, d), generator=gen, device=DEV)).bfloat16()
    over = any(n > length for length, n in zip(lens, news))
    want, want_lse = reference(q, cache, table, lens, news, frame, window, sink)
    cache, table = hide(cache, table, lens, news, frame, window, sink)
    ws = torch.full((1 << 26,), 0xA5, dtype=torch.uint8, device=DEV)
    out, lse = sa.cache_fwd(q, cache, table, kv_len, q_start=q_start, max_new=max(news), frame_tokens=frame, window=window, sink=sink, return_lse=True,
                            workspace=ws)
    assert sa.read_status(ws) == (sa.E_BAD_INDEX if over else sa.OK)
    check(out, lse, want, want_lse)


def call(q, cache, table, lens, news, **more):
    kv_len, q_start = batch_of(lens, news)
    return sa.cache_fwd(q, cache, table, kv_len, q_start=q_start, max_new=max(news), return_lse=True, check_status=True, **more)


@pytest.mark.parametrize("news", [[1, 1], [5, 30], [200, 90]])
def test_none_of_them_is_the_window_alone(news):
    """No first tokens, a window that holds them anyhow, no window: the same bits as the call without."""
    gen = torch.Generator(device=DEV).manual_seed(5)
    lens = [700, 333]
    cache = make_cache(gen, 40, 2, 32, 128, True)
    table = make_table(gen, lens, 32, 40)
    q = torch.randn((sum(news), 4, 128), generator=gen, device=DEV).bfloat16()
    for with_, without in ((dict(window=50, sink=0), dict(window=50)), (dict(window=0, sink=9), dict(window=0)), (dict(frame_tokens=0, sink=9), dict(frame_tokens=0)),
                           (dict(window=2 ** 31 - 1, sink=9), dict(window=0))):
        for x, y in zip(call(q, cache, table, lens, news, **with_), call(q, cache, table, lens, news, **without)):
            assert same_bits(x, y)
    for x, y in zip(call(q, cache, table, lens, news, window=20, sink=2 ** 31 - 1), call(q, cache, table, lens, news, window=0)):
        assert (x.double() - y.double()).abs().max() <= 2e-2 * y.double().abs().max()


@pytest.mark.parametrize("fp8", [True, False])
@pytest.mark.parametrize("news,G", [([1, 1, 1], 3), ([4, 2, 1], 4), ([30, 17, 1], 4), ([300, 129, 40], 1)])
def test_a_broken_value_reaches_the_rows_that_see_it(fp8, news, G):
    """A NaN among the first tokens, one in the window and one between them."""
    gen = torch.Generator(device=DEV).manual_seed(11)
    lens, Hk, page, frame, window, sink = [900, 400, 64], 2, 64, 1, 150, 21
    pages = sum(-(-n // page) for n in lens) + 1
    cache = make_cache(gen, pages, Hk, page, 128, fp8)
    table = make_table(gen, lens, page, pages)
    q = torch.randn((sum(news), Hk * G, 128), generator=gen, device=DEV).bfloat16()
    clean = call(q, cache, table, lens, news, window=window, sink=sink)
    for b, j in ((0, 7), (0, 20), (0, 21), (0, 700), (0, 880), (1, 0), (1, 395), (2, 63), (2, 30)):
        broken = cache.v.clone()
        page_of, slot = int(table[b, j // page]), j % page
        broken.view(torch.uint8 if fp8 else torch.int16)[page_of, 1, slot, 5] = 0x7f if fp8 else 0x7fc0
        out, lse = call(q, cache._replace(v=broken), table, lens, news, window=window, sink=sink)
        start = sum(news[:b])
        rows = [start + i for i in range(news[b]) if j in seen_keys(lens[b] - news[b] + i, lens[b], frame, window, sink)]
        hit = torch.zeros(out.shape, dtype=torch.bool, device=DEV)
        hit[rows, G:2 * G, 5] = True
        assert torch.equal(torch.isnan(out), hit)
        assert same_bits(lse, clean[1]) and torch.equal(torch.where(hit, 0, out), torch.where(hit, 0, clean[0]))


def test_captured_and_replayed_while_a_stream_goes_on():
    """One captured call for every step of a sequence that goes on past its window: lengths and table change under it."""
    gen = torch.Generator(device=DEV).manual_seed(3)
    Hk, page, d, window, sink = 2, 16, 128, 40, 20
    cache = make_cache(gen, 30, Hk, page, d, True)
    table = torch.full((1, 25), -1, dtype=torch.int32, device=DEV)
    kv_len = torch.ones(1, dtype=torch.int32, device=DEV)
    q = torch.randn((1, 4, d), generator=gen, device=DEV).bfloat16()
    full = torch.randperm(30, generator=gen, device=DEV).int()[:25][None]
    table.copy_(full)
    ws = torch.empty(1 << 24, dtype=torch.uint8, device=DEV)
    out = torch.empty_like(q)
    args = dict(window=window, sink=sink, out=out, workspace=ws)
    sa.cache_fwd(q, cache, table, kv_len, **args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sa.cache_fwd(q, cache, table, kv_len, **args)
    for n in (1, 20, 41, 61, 62, 200, 399):
        kv_len.fill_(n)
        gone = full.clone()
        gone[:, 2:max(n - window, 0) // page] = -1
        table.copy_(gone if max(n - window, 0) // page > 2 else full)
        graph.replay()
        assert sa.read_status(ws) == sa.OK
        want, lse = reference(q, cache, full, [n], [1], 1, window, sink)
        got = out.double()
        assert (got - want).abs().max() <= 1.2e-2 * want.abs().max()


def test_a_page_that_is_seen_and_is_not_there_is_reported():
    gen = torch.Generator(device=DEV).manual_seed(3)
    cache = make_cache(gen, 30, 1, 16, 64, True)
    for news in (1, 40):
        q = torch.randn((news, 1, 64), generator=gen, device=DEV).bfloat16()
        kv_len = torch.tensor([400], dtype=torch.int32, device=DEV)
        for entry, bad in ((0, True), (1, True), (2, False), (15, False), (24, True), (25, False)):
            table = torch.arange(26, dtype=torch.int32, device=DEV)[None].contiguous()
            table[0, entry] = 30
            ws = torch.zeros(1 << 24, dtype=torch.uint8, device=DEV)
            out = sa.cache_fwd(q, cache, table, kv_len, max_new=news, window=60, sink=20, workspace=ws)
            assert sa.read_status(ws) == (sa.E_BAD_INDEX if bad else sa.OK)
            assert torch.isfinite(out).all()


ROW_TILES = [
    # lens, news, H, Hk, d, page, fp8, frame, window, sink: 17 to 128 rows per key head
    ([900, 907], [5, 5], 16, 2, 128, 64, True, 1, 90, 21),
    ([900, 907], [5, 5], 16, 2, 128, 64, False, 1, 90, 21),
    ([900, 0, 7, 300], [5, 0, 1, 3], 8, 1, 64, 16, True, 1, 70, 4),       # sequences with fewer row tiles, and with none
    ([900, 0, 7, 300], [5, 0, 1, 3], 8, 1, 64, 16, False, 1, 70, 129),
    ([700, 650, 700], [17, 2, 16], 2, 2, 128, 32, True, 1, 40, 1),        # tiles of one row, of sixteen
    ([700, 650], [33, 32], 2, 2, 128, 128, False, 1, 300, 64),
    ([1300, 5], [9, 4], 24, 2, 128, 16, True, 1, 200, 500),
    ([900], [128], 3, 3, 64, 64, True, 1, 77, 10),
    ([900, 800], [60, 20], 4, 2, 128, 64, True, 25, 2, 25),               # rows of several frames in a tile
    ([6000], [7], 12, 1, 128, 64, True, 1, 3000, 4),
    ([20000], [9], 5, 1, 64, 128, False, 1, 12000, 300),
    ([3, 130, 513], [7, 30, 1], 14, 7, 128, 64, True, 1, 50, 3),          # more new tokens than the first sequence holds
]


@pytest.mark.parametrize("case", ROW_TILES, ids=lambda c: "-".join(str(x) for x in c[2:]) + f"-{len(c[0])}x{max(c[0])}")
@pytest.mark.parametrize("spare", [1, 700])
def test_row_tiles(case, spare):
    test_window_and_first_tokens(case, spare)


def test_row_tiles_captured():
    """A graph that holds two such calls, replayed with other lengths and queries, some sequences without rows."""
    gen = torch.Generator(device=DEV).manual_seed(21)
    lens, news, Hk, G, page = [600, 444, 90], [6, 6, 6], 2, 6, 32
    pages = sum(-(-n // page) for n in lens) + 2
    cache = make_cache(gen, pages, Hk, page, 128, True)
    table = make_table(gen, lens, page, pages)
    kv_len, q_start = batch_of(lens, news)
    q = torch.randn((sum(news), Hk * G, 128), generator=gen, device=DEV).bfloat16()
    args = dict(q_start=q_start, max_new=6, return_lse=True)
    outs = [None, None]

    def step():
        outs[0] = sa.cache_fwd(q, cache, table, kv_len, window=60, sink=5, **args)
        outs[1] = sa.cache_fwd(q, cache, table, kv_len, window=200, sink=70, **args)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for lens, news in (([600, 444, 90], [6, 6, 6]), ([580, 0, 33], [3, 0, 6]), ([64, 100, 90], [1, 6, 0])):
        a, b = batch_of(lens, news)
        kv_len.copy_(a)
        q_start.copy_(b)
        q.copy_(torch.randn(q.shape, generator=gen, device=DEV))
        graph.replay()
        n = sum(news)
        for (out, lse), (window, sink) in zip(outs, ((60, 5), (200, 70))):
            want, want_lse = reference(q[:n], cache, table, lens, news, 1, window, sink)
            check(out[:n], lse[:n], want, want_lse)
