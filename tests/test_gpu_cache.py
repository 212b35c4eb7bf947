"""GPU parity of the paged cache: appending with rotation (bit-exact against a restatement in plain torch operations) and
attention over bf16 and E4M3 pages against softmax attention in 64 bits on the very values that the pages hold."""
import math

import pytest
import torch

import paper_2609_23153_b200 as sa

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

# Bounds, from the roundings between the inputs and the result.  out is rounded to bf16 (2^-9 of a value) and the weights to bf16 (bf16
# pages, many rows) or fp16: relative RMS at most 2^-9 / sqrt(3) from each, 1.6e-3 together; where few keys dominate, a row's own
# error may reach the sum of two full roundings.  lse: fp32 products and sums over at most 128 channels and the exponential's 2^-22.
OUT_RELRMS, OUT_MAX_OF_ROW, LSE_ABS = 2.5e-3, 1.2e-2, 2e-4


def make_cache(gen, pages, heads, page, d, fp8, general=False, layout="hnd"):
    """A pool filled with normal values; E4M3 scales are powers of two, or any positive number (`general`)."""
    shape = (pages, heads, page, d) if layout == "hnd" else (pages, page, heads, d)
    k, v = (torch.randn(shape, generator=gen, device=DEV) * torch.exp(torch.randn((1, 1, 1, d), generator=gen, device=DEV) * 0.5) for _ in range(2))
    if not fp8:
        c = [x.bfloat16() for x in (k, v)]
    else:
        c = [x.mul(60.0).clamp(-448, 448).to(torch.float8_e4m3fn) for x in (k, v)]
    if layout != "hnd":
        c = [x.transpose(1, 2) for x in c]
    if not fp8:
        return sa.KVCache(*c)
    s = [torch.exp2(torch.randint(-8, -4, (pages, heads), generator=gen, device=DEV).float()) for _ in range(2)]
    if general:
        s = [x * (1 + torch.rand((pages, heads), generator=gen, device=DEV)) for x in s]
    return sa.KVCache(*c, *s)


def make_table(gen, lens, page, pages, spare=1):
    """Every sequence's pages in a random order, and columns that nothing may read."""
    need = [-(-n // page) for n in lens]
    order = torch.randperm(pages, generator=gen, device=DEV).int()
    table = torch.full((len(lens), max(need) + spare), -7, dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    assert at <= pages
    return table


def batch_of(lens, news):
    starts = [0]
    for n in news:
        starts.append(starts[-1] + n)
    return torch.tensor(lens, dtype=torch.int32, device=DEV), torch.tensor(starts, dtype=torch.int32, device=DEV)


def visible(pos, length, frame, window):
    if frame == 0:
        return 0, length
    if pos < 0:
        return 0, 0
    f = pos // frame
    return (max(0, (f - window + 1) * frame) if window else 0), min(length, (f + 1) * frame)


def reference(q, cache, table, lens, news, frame, window, scale=None):
    """Softmax attention in 64 bits, row by row over exactly the keys that a row sees."""
    Hk, P, d = cache.k.shape[1:]
    T, H, _ = q.shape
    G = H // Hk
    out = torch.zeros((T, H, d), dtype=torch.float64, device=DEV)
    lse = torch.full((T, H), -math.inf, dtype=torch.float64, device=DEV)
    t = 0
    for b, (length, n) in enumerate(zip(lens, news)):
        pages = table[b, :-(-length // P)].long()
        for i in range(n):
            lo, hi = visible(length - n + i, length, frame, window)
            if hi > lo:
                first, last = lo // P, -(-hi // P)
                pg = pages[first:last]
                def rows(x, s):
                    y = x.view(torch.uint8)[pg].view(torch.float8_e4m3fn).double() if s is not None else x[pg].double()
                    y = y if s is None else y * s[pg].double()[:, :, None, None]
                    return y.transpose(0, 1).reshape(Hk, -1, d)[:, lo - first * P:hi - first * P]
                kk, vv = rows(cache.k, cache.k_scale), rows(cache.v, cache.v_scale)
                a = torch.einsum("hgd,hjd->hgj", q[t].double().view(Hk, G, d), kk) * (scale or d ** -0.5)
                lse[t] = torch.logsumexp(a, -1).view(H)
                out[t] = torch.einsum("hgj,hjd->hgd", torch.softmax(a, -1), vv).reshape(H, d)
            t += 1
    return out, lse


def check(got, lse, want, want_lse):
    got, lse = got.double(), lse.double()
    assert torch.isfinite(got).all()
    empty = torch.isinf(want_lse)
    assert torch.equal(torch.isinf(lse) & (lse < 0), empty)
    assert (got[empty] == 0).all()
    if empty.all():
        return
    rms = (got - want).square().mean().sqrt() / want.square().mean().sqrt()
    size = want.abs().amax(-1, keepdim=True).clamp(min=1e-6)
    worst = ((got - want).abs() / size)[~empty].max()
    off = (lse - want_lse)[~empty].abs().max()
    print(f"relrms {float(rms):.2e} worst {float(worst):.2e} lse {float(off):.2e}")
    assert rms <= OUT_RELRMS and worst <= OUT_MAX_OF_ROW and off <= LSE_ABS


CASES = [
    # lens, news, H, Hk, d, page, fp8, frame, window
    ([1], [1], 8, 8, 128, 16, True, 1, 0),
    ([17], [1], 4, 1, 64, 16, True, 1, 0),
    ([64, 65, 63], [1, 1, 1], 16, 2, 128, 64, True, 1, 0),
    ([1000, 1, 333, 128], [1, 1, 1, 1], 40, 8, 128, 64, True, 1, 0),
    ([2049, 7], [1, 1], 24, 2, 128, 32, False, 1, 0),
    ([700, 0, 31], [1, 1, 1], 12, 12, 64, 32, False, 1, 0),
    ([0, 0], [1, 2], 4, 4, 128, 16, True, 1, 0),
    ([900, 513], [3, 5], 16, 4, 128, 16, True, 1, 0),
    ([900, 513], [3, 5], 16, 4, 64, 128, True, 0, 0),
    ([411], [9], 32, 2, 128, 64, False, 1, 0),
    ([1500, 40, 77], [1, 1, 1], 16, 4, 64, 16, True, 1, 100),
    ([1500, 800], [1, 4], 6, 3, 128, 128, True, 50, 2),
    ([260, 2], [260, 2], 4, 2, 128, 64, True, 1, 0),
    ([330], [200], 3, 1, 64, 16, False, 64, 0),
    ([77, 500], [20, 300], 8, 8, 128, 32, True, 1, 33),
    ([5000], [1], 8, 1, 128, 128, True, 1, 0),
    ([40000, 100], [1, 1], 2, 2, 128, 64, True, 1, 0),
    ([600, 129, 1], [129, 128, 1], 1, 1, 128, 64, True, 1, 0),
    ([2000, 0, 515], [300, 4, 257], 8, 2, 128, 16, True, 1, 0),
    ([2000, 1600, 40], [40, 90, 17], 16, 1, 64, 128, True, 0, 0),
    ([1300, 900], [700, 300], 4, 4, 128, 128, True, 100, 3),
    ([1300, 900], [700, 300], 5, 5, 128, 32, False, 1, 256),
    ([7000], [40], 3, 1, 64, 64, False, 1, 0),
    ([9000, 8], [33, 8], 40, 8, 128, 64, True, 1, 0),
    ([3, 130, 513], [7, 130, 1], 7, 7, 128, 64, True, 1, 0),         # more new tokens than the first sequence holds
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) for x in c[2:]) + f"-{len(c[0])}x{max(c[0])}")
@pytest.mark.parametrize("general", [False, True])
def test_attention_over_pages(case, general):
    lens, news, H, Hk, d, page, fp8, frame, window = case
    if general and not fp8:
        pytest.skip("bf16 pages have no scales")
    gen = torch.Generator(device=DEV).manual_seed(sum(lens) + H)
    pages = sum(-(-n // page) for n in lens) + 2
    cache = make_cache(gen, pages, Hk, page, d, fp8, general, layout="nhd" if general else "hnd")
    table = make_table(gen, lens, page, pages)
    kv_len, q_start = batch_of(lens, news)
    q = (1.5 * torch.randn((sum(news), H, d), generator=gen, device=DEV)).bfloat16()
    over = any(n > length for length, n in zip(lens, news))
    ws = torch.full((1 << 26,), 0xA5, dtype=torch.uint8, device=DEV)
    out, lse = sa.cache_fwd(q, cache, table, kv_len, q_start=q_start, max_new=max(news), frame_tokens=frame, window=window,
                            return_lse=True, workspace=ws)
    assert sa.read_status(ws) == (sa.E_BAD_INDEX if over else sa.OK)
    want, want_lse = reference(q, cache, table, lens, news, frame, window)
    check(out, lse, want, want_lse)


# ------------------------------------------------------------------------------------------------------------------ append

def power_scale(amax):
    m, e = torch.frexp(amax.clamp(min=1e-12))
    return torch.ldexp(torch.ones_like(amax), e - 9 + (m > 0.875).int())


def encode(x):
    return x.clamp(-448, 448).to(torch.float8_e4m3fn)


def turned(x, c, s, interleaved):
    rot = 2 * c.numel()
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    y = x.clone()
    p, r = a * c - b * s, a * s + b * c
    if interleaved:
        y[..., 0:rot:2], y[..., 1:rot:2] = p, r
    else:
        y[..., :rot // 2], y[..., rot // 2:rot] = p, r
    return y


def append_reference(cache, k, v, table, lens, news, rotary, q):
    """Token by token, page by page, in 32 bits.  Runs on the CPU."""
    cpu = lambda x: None if x is None else x.cpu()
    kc, vc, ks, vs = (None if x is None else x.cpu().clone() for x in cache)
    k, v, q, table = k.cpu().float(), v.cpu().float(), cpu(q), table.cpu()
    q = None if q is None else q.float()
    P = kc.shape[2]
    fp8 = ks is not None
    t = 0
    for b, (length, n) in enumerate(zip(lens, news)):
        if rotary is not None:
            cos, sin, positions, axis, inter = (cpu(x) if isinstance(x, torch.Tensor) else x for x in rotary)
            m = torch.arange(cos.shape[1])
            for i in range(n):
                at = torch.full_like(m, length - n + i)
                if positions is not None:
                    at = positions.view(len(positions), -1)[t + i].long()[axis.long() if axis is not None else torch.zeros_like(m)]
                k[t + i] = turned(k[t + i], cos[at, m], sin[at, m], inter)
                if q is not None:
                    q[t + i] = turned(q[t + i], cos[at, m], sin[at, m], inter)
        pos = length - n
        i = 0
        while i < n:
            page, slot = int(table[b, (pos + i) // P]), (pos + i) % P
            m = min(P - slot, n - i)
            for x, pool, scale in ((k, kc, ks), (v, vc, vs)):
                new = x[t + i:t + i + m].transpose(0, 1)
                if fp8:
                    amax = torch.where(torch.isfinite(new), new.abs(), 0.0).amax(dim=(1, 2))
                    fit = power_scale(amax)
                    if slot > 0:
                        fit = torch.maximum(fit, scale[page])
                        again = encode(pool[page, :, :slot].float() * (scale[page] * (1.0 / fit))[:, None, None])
                        grew = (fit > scale[page])[:, None, None]
                        pool.view(torch.uint8)[page, :, :slot] = torch.where(grew, again.view(torch.uint8), pool.view(torch.uint8)[page, :, :slot])
                    scale[page] = fit
                    pool.view(torch.uint8)[page, :, slot:slot + m] = encode(new * (1.0 / fit)[:, None, None]).view(torch.uint8)
                else:
                    pool[page, :, slot:slot + m] = new.bfloat16()
            i += m
        t += n
    return sa.KVCache(kc, vc, ks, vs), None if q is None else q.bfloat16()


def same_bits(a, b):
    view = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[a.element_size()]
    return torch.equal(a.cpu().contiguous().view(view), b.cpu().contiguous().view(view))


def make_rotary(gen, d, rot, rows, T, axes, interleaved):
    angle = torch.rand((rows, rot // 2), generator=gen, device=DEV) * 6.3
    positions = axis = None
    if axes > 0:
        positions = torch.randint(0, rows, (T, axes), generator=gen, device=DEV).int()
        axis = torch.randint(0, axes, (rot // 2,), generator=gen, device=DEV).int()
    return sa.Rotary(angle.cos(), angle.sin(), positions, axis, interleaved)


APPENDS = [
    # lens, news, H, Hk, d, page, fp8, rot, axes, interleaved
    ([1], [1], 8, 8, 128, 16, True, 128, 0, False),
    ([64, 65, 190], [1, 1, 1], 40, 8, 128, 64, True, 64, 0, False),
    ([5, 17, 33, 64], [5, 3, 16, 1], 6, 2, 64, 16, True, 64, 0, True),
    ([300, 130], [300, 129], 4, 4, 128, 128, True, 128, 3, True),
    ([300, 130], [290, 130], 3, 1, 128, 64, False, 32, 0, False),
    ([77], [70], 2, 2, 64, 32, False, 64, 2, False),
    ([200, 9, 1], [100, 2, 1], 5, 5, 64, 128, True, 16, 0, False),
    ([200, 90], [37, 33], 16, 4, 128, 32, True, 0, 0, False),
    ([1000, 40], [2, 4], 8, 1, 128, 128, True, 128, 1, False),
]


@pytest.mark.parametrize("case", APPENDS, ids=lambda c: "-".join(str(x) for x in c[2:]) + f"-{len(c[0])}x{max(c[1])}")
@pytest.mark.parametrize("layout", ["hnd", "nhd"])
def test_append_bits(case, layout):
    lens, news, H, Hk, d, page, fp8, rot, axes, interleaved = case
    gen = torch.Generator(device=DEV).manual_seed(sum(lens) + d)
    pages = sum(-(-n // page) for n in lens) + 2
    cache = make_cache(gen, pages, Hk, page, d, fp8, layout=layout)
    table = make_table(gen, lens, page, pages)
    kv_len, q_start = batch_of(lens, news)
    T = sum(news)
    # fused projections: q, k and v are parts of the same rows
    qkv = torch.randn((T, H + 2 * Hk, d), generator=gen, device=DEV) * torch.exp(1.5 * torch.randn((T, 1, 1), generator=gen, device=DEV))
    qkv = qkv.bfloat16()
    q, k, v = qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:]
    rotary = make_rotary(gen, d, rot, max(lens), T, axes, interleaved) if rot else None
    want, want_q = append_reference(cache, k, v, table, lens, news, rotary, q)
    ws = torch.full((256,), 0xA5, dtype=torch.uint8, device=DEV)
    got_q = sa.cache_append(cache, k, v, table, kv_len, q_start=q_start, max_new=max(news), q=q, rotary=rotary, workspace=ws)
    assert sa.read_status(ws) == sa.OK
    assert same_bits(got_q, want_q)
    for got, ref in zip(cache, want):
        assert (got is None) == (ref is None)
        if got is not None:
            assert same_bits(got, ref)
    again = sa.cache_append(cache, k, v, table, kv_len, q_start=q_start, max_new=max(news), q=q, q_out=q, rotary=rotary)
    assert again.data_ptr() == q.data_ptr() and same_bits(again, want_q)         # in place, and appending again changes nothing
    for got, ref in zip(cache, want):
        assert got is None or same_bits(got, ref)


# ------------------------------------------------------------------------------------------------- what must not be looked at

def poisoned(cache, table, lens, page):
    """The cache with NaN, infinities and the type's largest values wherever no sequence has a token: behind the last token of a page,
    and in pages of nobody."""
    fp8 = cache.k_scale is not None
    owned = torch.zeros((cache.k.shape[0], page), dtype=torch.bool, device=DEV)
    for b, n in enumerate(lens):
        for i in range(-(-n // page)):
            owned[int(table[b, i]), :min(page, n - i * page)] = True
    junk = torch.tensor([0x7f, 0xff, 0x7e, 0xfe] if fp8 else [0x7fc0, -0x0080, 0x7f80, 0x7f7f], device=DEV)
    out = []
    for x in (cache.k, cache.v):
        bits = x.view(torch.uint8 if fp8 else torch.int16).clone(memory_format=torch.preserve_format)
        pattern = junk[torch.arange(bits.numel(), device=DEV) % 4].view(bits.shape).to(bits.dtype)
        bits = torch.where(owned[:, None, :, None], bits, pattern)
        out.append(bits.view(x.dtype))
    scales = []
    for s in (cache.k_scale, cache.v_scale):
        if s is not None:
            s = s.clone()
            s[~owned.any(1)] = math.nan
        scales.append(s)
    return sa.KVCache(*out, *scales)


@pytest.mark.parametrize("fp8", [True, False])
@pytest.mark.parametrize("d,page,G,news", [(128, 64, 1, [1, 1, 1]), (128, 16, 4, [3, 2, 4]), (64, 128, 2, [1, 1, 1]), (128, 128, 2, [60, 1, 17]),
                                           (64, 32, 3, [200, 5, 90]), (128, 32, 4, [150, 31, 2])])
def test_nothing_behind_the_last_token(fp8, d, page, G, news):
    gen = torch.Generator(device=DEV).manual_seed(page + G)
    lens, Hk = [517, 33, 260], 3
    pages = sum(-(-n // page) for n in lens) + 4
    cache = make_cache(gen, pages, Hk, page, d, fp8, general=fp8)
    table = make_table(gen, lens, page, pages, spare=3)
    kv_len, q_start = batch_of(lens, news)
    q = torch.randn((sum(news), Hk * G, d), generator=gen, device=DEV).bfloat16()
    for frame, window in ((1, 0), (1, 70), (0, 0), (40, 2)):
        want = sa.cache_fwd(q, cache, table, kv_len, q_start=q_start, max_new=max(news), frame_tokens=frame, window=window, return_lse=True)
        got = sa.cache_fwd(q, poisoned(cache, table, lens, page), table, kv_len, q_start=q_start, max_new=max(news), frame_tokens=frame,
                           window=window, return_lse=True, check_status=True)
        assert all(torch.isfinite(x).all() for x in want)
        assert all(same_bits(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("fp8", [True, False])
@pytest.mark.parametrize("d,G,n,length", [(128, 2, 4, 300), (64, 4, 4, 150), (128, 1, 200, 500), (128, 4, 100, 257), (64, 1, 300, 300), (128, 2, 40, 128)])
@pytest.mark.parametrize("frame,window", [(1, 0), (1, 40), (16, 2)])
def test_values_that_are_not_finite_reach_only_who_sees_them(fp8, d, G, n, length, frame, window):
    """NaN and infinities in keys and values: the rows that see such a key have what the formula gives (NaN in the channels of a value,
    everywhere for a key), all others are bit for bit what they are without."""
    gen = torch.Generator(device=DEV).manual_seed(n + d)
    page, Hk = 32, 2
    pages = -(-length // page)
    cache = make_cache(gen, pages, Hk, page, d, fp8)
    table = make_table(gen, [length], page, pages)
    kv_len, q_start = batch_of([length], [n])
    q = torch.randn((n, Hk * G, d), generator=gen, device=DEV).bfloat16()
    kw = dict(q_start=q_start, max_new=n, frame_tokens=frame, window=window, return_lse=True)
    clean, clean_lse = sa.cache_fwd(q, cache, table, kv_len, **kw)
    marks = [(length - 1, 3, math.nan), (length - n // 2, 5, math.nan), (length - n // 2, 9, math.inf), (max(0, length - n - 20), 1, -math.inf),
             (length - n // 2 - 1, 9, -math.inf)]
    bad_key = length - n // 3 - 1
    k, v = (x.clone(memory_format=torch.preserve_format) for x in cache[:2])

    def put(x, j, h, c, value):
        at = (int(table[0, j // page]), h, j % page, c)
        if fp8:
            x.view(torch.uint8)[at] = 0x7f                    # E4M3 has no infinity
        else:
            x[at] = value
    for j, c, value in marks:
        put(v, j, 0, c, value)
    put(k, bad_key, 1, 7, math.nan)
    got, lse = sa.cache_fwd(q, sa.KVCache(k, v, *cache[2:]), table, kv_len, **kw)
    want, want_lse = clean.float(), clean_lse.clone()
    for i in range(n):
        lo, hi = visible(length - n + i, length, frame, window)
        for j, c, value in marks:
            if lo <= j < hi:
                want[i, :G, c] += math.nan if fp8 else value
        if lo <= bad_key < hi:
            want[i, G:] = math.nan
            want_lse[i, G:] = math.nan
    want = want.bfloat16()
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.isnan(lse), torch.isnan(want_lse))
    assert same_bits(torch.where(torch.isnan(want), 0.0, got), torch.where(torch.isnan(want), 0.0, want))
    fine = ~torch.isnan(want_lse)
    assert same_bits(lse[fine], want_lse[fine])


def test_pages_that_do_not_exist():
    """A page number outside the pool: reported, its tokens are not attended to and not stored."""
    gen = torch.Generator(device=DEV).manual_seed(5)
    for n, H in ((1, 4), (40, 4)):
        lens = [300, 200]
        cache = make_cache(gen, 12, 2, 64, 128, True)
        table = make_table(gen, lens, 64, 12)
        kv_len, q_start = batch_of(lens, [n, n])
        q = torch.randn((2 * n, H, 128), generator=gen, device=DEV).bfloat16()
        broken = table.clone()
        broken[0, 1], broken[1, 0] = 12, -1
        ws = torch.empty(1 << 26, dtype=torch.uint8, device=DEV)
        out, lse = sa.cache_fwd(q, cache, broken, kv_len, q_start=q_start, max_new=n, frame_tokens=0, return_lse=True, workspace=ws)
        assert sa.read_status(ws) == sa.E_BAD_INDEX
        # the same without those keys: they become the last ones, behind the length
        for b, gone in ((0, 1), (1, 0)):
            keep = [i for i in range(-(-lens[b] // 64)) if i != gone]
            t2 = table[b:b + 1, keep].contiguous()
            want, want_lse = sa.cache_fwd(q[b * n:(b + 1) * n], cache, t2, kv_len[b:b + 1] - 64, max_new=n, frame_tokens=0, return_lse=True, workspace=ws)
            assert sa.read_status(ws) == sa.OK
            assert (out[b * n:(b + 1) * n].float() - want.float()).abs().max() <= 2 ** -7 * want.float().abs().max()
            assert (lse[b * n:(b + 1) * n] - want_lse).abs().max() <= 1e-4
        before = [x.clone() for x in cache]
        k = torch.randn((2 * n, 2, 128), generator=gen, device=DEV).bfloat16()
        broken[:] = 99
        sa.cache_append(cache, k, k, broken, kv_len, q_start=q_start, max_new=n, workspace=ws)
        assert sa.read_status(ws) == sa.E_BAD_INDEX
        assert all(same_bits(x, y) for x, y in zip(cache, before))


@pytest.mark.parametrize("what", ["negative length", "length beyond the table", "starts descend", "starts beyond the rows", "more than max_new"])
def test_numbers_that_do_not_fit_stay_inside(what):
    """Device-side numbers of a broken caller: reported, and nothing outside the tensors is touched (the call ends, its neighbours' pages
    keep their bits)."""
    gen = torch.Generator(device=DEV).manual_seed(6)
    cache = make_cache(gen, 8, 2, 16, 64, True)
    table = make_table(gen, [40, 50], 16, 8, spare=0)
    lens, starts = [40, 50], [0, 3, 6]
    if what == "negative length":
        lens[0] = -5
    elif what == "length beyond the table":
        lens[1] = 100000
    elif what == "starts descend":
        starts = [4, 2, 6]
    elif what == "starts beyond the rows":
        starts = [0, 3, 900]
    kv_len = torch.tensor(lens, dtype=torch.int32, device=DEV)
    q_start = torch.tensor(starts, dtype=torch.int32, device=DEV)
    q = torch.randn((6, 4, 64), generator=gen, device=DEV).bfloat16()
    max_new = 2 if what == "more than max_new" else 3
    ws = torch.empty(1 << 26, dtype=torch.uint8, device=DEV)
    sa.cache_fwd(q, cache, table, kv_len, q_start=q_start, max_new=max_new, workspace=ws)
    assert sa.read_status(ws) == sa.E_BAD_INDEX
    k = q[:, :2].contiguous()
    sa.cache_append(cache, k, k, table, kv_len, q_start=q_start, max_new=max_new, q=q, workspace=ws)
    assert sa.read_status(ws) == sa.E_BAD_INDEX


# --------------------------------------------------------------------------------------------------------- shapes of memory

@pytest.mark.parametrize("news", [[1], [30]])
def test_offsets_beyond_32_bits(news):
    """A pool of 2.7 billion entries per side, whose last pages hold the sequence."""
    pages, Hk, page, d = 41000, 8, 64, 128
    pools = [torch.empty((pages, Hk, page, d), dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn) for _ in range(2)]
    scales = [torch.ones((pages, Hk), device=DEV) for _ in range(2)]
    gen = torch.Generator(device=DEV).manual_seed(9)
    lens = [333]
    table = torch.arange(pages - 6, pages, device=DEV, dtype=torch.int32)[None].contiguous()
    kv_len, q_start = batch_of(lens, lens)
    k, v = (torch.randn((333, Hk, d), generator=gen, device=DEV).bfloat16() for _ in range(2))
    cache = sa.KVCache(*pools, *scales)
    sa.cache_append(cache, k, v, table, kv_len, q_start=q_start, max_new=333, check_status=True)
    small = sa.KVCache(*(x[-6:].clone() for x in cache))
    check_k = small.k.view(torch.uint8).view(torch.float8_e4m3fn).float() * small.k_scale[:, :, None, None]
    got = check_k.transpose(1, 2).reshape(-1, Hk, d)[:333]
    assert (got - k.float()).abs().max() <= 2 ** -4 * k.float().abs().max()
    q = torch.randn((news[0], 16, d), generator=gen, device=DEV).bfloat16()
    a = sa.cache_fwd(q, cache, table, kv_len, check_status=True)
    b = sa.cache_fwd(q, small, table - (pages - 6), kv_len, check_status=True)
    assert same_bits(a, b)


@pytest.mark.parametrize("n", [1, 3, 50])
def test_views_streams_and_defaults(n):
    """Rows of fused projections, an output inside a larger tensor, equal shares without q_start, another stream, a captured graph
    whose lengths change between replays: the same bits every time."""
    gen = torch.Generator(device=DEV).manual_seed(11)
    B, Hk, G, page, d = 3, 2, 3, 32, 128
    lens = [200, 77, 130]
    cache = make_cache(gen, 30, Hk, page, d, True)
    table = make_table(gen, [256] * 3, page, 30)
    kv_len, q_start = batch_of(lens, [n] * B)
    rows = torch.randn((B * n, 20, d), generator=gen, device=DEV).bfloat16()
    q = rows[:, 4:4 + Hk * G]
    want, want_lse = sa.cache_fwd(q.contiguous(), cache, table, kv_len, q_start=q_start, max_new=n, return_lse=True)
    room = torch.zeros((B * n, 3, Hk * G, d), dtype=torch.bfloat16, device=DEV)
    got = sa.cache_fwd(q, cache, table, kv_len, out=room[:, 1])
    assert got.data_ptr() == room[:, 1].data_ptr() and same_bits(got, want)
    assert (room[:, 0] == 0).all() and (room[:, 2] == 0).all()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    x, lse = sa.cache_fwd(q, cache, table, kv_len, stream=side, return_lse=True, max_new=n)
    side.synchronize()
    assert same_bits(x, want) and same_bits(lse, want_lse)
    graph = torch.cuda.CUDAGraph()
    length = kv_len.clone()
    ws = torch.empty(1 << 26, dtype=torch.uint8, device=DEV)
    out = torch.empty_like(want)
    with torch.cuda.graph(graph):
        sa.cache_fwd(q, cache, table, length, out=out, workspace=ws)
    for lens2 in ([200, 77, 130], [60, 256, 51], [200, 77, 130]):
        length.copy_(torch.tensor(lens2, dtype=torch.int32, device=DEV))
        graph.replay()
        want2 = sa.cache_fwd(q, cache, table, length)
        assert same_bits(out, want2) and sa.read_status(ws) == sa.OK


def test_many_short_sequences():
    """More sequences than CTAs, lengths from zero on, one to three new tokens."""
    gen = torch.Generator(device=DEV).manual_seed(12)
    B = 700
    news = [1 + i % 3 for i in range(B)]
    lens = [max(news[i], (i * 7) % 40) if i % 11 else 0 for i in range(B)]
    news = [min(n, max(length, 1)) for n, length in zip(news, lens)]
    pages = sum(-(-n // 16) for n in lens) + 1
    cache = make_cache(gen, pages, 2, 16, 64, True)
    table = make_table(gen, lens, 16, pages)
    kv_len, q_start = batch_of(lens, news)
    for H in (2, 12, 64):
        q = torch.randn((sum(news), H, 64), generator=gen, device=DEV).bfloat16()
        out, lse = sa.cache_fwd(q, cache, table, kv_len, q_start=q_start, max_new=3, return_lse=True)
        want, want_lse = reference(q, cache, table, lens, news, 1, 0)
        check(out, lse, want, want_lse)


@pytest.mark.parametrize("scale", [0.02, 1.7])
def test_softmax_scale_and_sharp_rows(scale):
    """A scale of the caller's, and logits far apart: one key takes nearly everything, others underflow."""
    gen = torch.Generator(device=DEV).manual_seed(13)
    for n in (1, 20):
        cache = make_cache(gen, 40, 2, 32, 128, True, general=True)
        lens, news = [900], [n]
        table = make_table(gen, lens, 32, 40)
        kv_len, q_start = batch_of(lens, news)
        q = (3 * torch.randn((n, 4, 128), generator=gen, device=DEV)).bfloat16()
        out, lse = sa.cache_fwd(q, cache, table, kv_len, softmax_scale=scale, return_lse=True, check_status=True)
        want, want_lse = reference(q, cache, table, lens, news, 1, 0, scale)
        rms = (out.double() - want).square().mean().sqrt() / want.square().mean().sqrt()
        # logits of up to a few thousand carry fp32's rounding: 2^-22 of the largest
        tol = 2 ** -22 * float(want_lse.abs().max()) * 16
        print(float(rms), float((lse - want_lse).abs().max()), tol)
        assert rms <= OUT_RELRMS + 2 * tol and (lse - want_lse).abs().max() <= LSE_ABS + tol


# --------------------------------------------------------------------------------------------------- how a page fills up

@pytest.mark.parametrize("fp8", [True, False])
@pytest.mark.parametrize("steps", [[1] * 40, [7, 1, 20, 3, 9], [40]])
def test_a_page_hardly_depends_on_its_steps(fp8, steps):
    """Token by token or at once: each way is the restatement's bits, and with power-of-two scales what they hold differs only where
    small values had been rounded to a larger scale's subnormal numbers before."""
    gen = torch.Generator(device=DEV).manual_seed(21)
    Hk, page, d, total = 3, 16, 64, 40
    k, v = (torch.randn((total, Hk, d), generator=gen, device=DEV) * torch.exp(torch.randn((total, Hk, 1), generator=gen, device=DEV) * 1.5) for _ in range(2))
    k, v = k.bfloat16(), v.bfloat16()
    k[5, 0, 3], k[6, 1, 0], v[11, 2, 1] = math.inf, math.nan, -math.inf
    cache = sa.alloc_cache(4, Hk, page, d, fp8=fp8)
    table = torch.tensor([[2, 0, 3]], dtype=torch.int32, device=DEV)
    want = sa.KVCache(*(None if x is None else x.clone() for x in cache))
    at = 0
    for n in steps:
        at += n
        kv_len = torch.tensor([at], dtype=torch.int32, device=DEV)
        sa.cache_append(cache, k[at - n:at], v[at - n:at], table, kv_len, check_status=True)
        want, _ = append_reference(want, k[at - n:at], v[at - n:at], table, [at], [n], None, None)
        for got, ref in zip(cache, want):
            if got is not None and got.dtype == torch.float32:
                assert same_bits(got, ref)
            elif got is not None:      # NaN is NaN, whichever
                a, b = got.cpu().float(), ref.float()
                assert torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(torch.nan_to_num(a, 0.0), torch.nan_to_num(b, 0.0))
    if fp8:
        whole = sa.alloc_cache(4, Hk, page, d)
        sa.cache_append(whole, k, v, table, torch.tensor([total], dtype=torch.int32, device=DEV))
        for a, b, s, t in ((cache.k, whole.k, cache.k_scale, whole.k_scale), (cache.v, whole.v, cache.v_scale, whole.v_scale)):
            assert torch.equal(s[[2, 0, 3]], t[[2, 0, 3]])
            x, y = (torch.nan_to_num(z.float(), 0.0) * s[:, :, None, None] for z in (a, b))
            # (an infinity became the largest number of the scale at its time)
            x, y = (torch.where(b.float().abs() == 448, 0.0, z) for z in (x, y))
            assert ((x - y).abs() <= s[:, :, None, None] * 2.0 ** -9).all()          # half a subnormal step twice


def test_append_then_attend_is_attention():
    """The two calls together, token by token, against softmax attention in 64 bits over the rotated bf16 values: bf16 pages exactly those
    values, E4M3 pages within the codes' rounding."""
    gen = torch.Generator(device=DEV).manual_seed(31)
    H, Hk, d, page, total = 4, 2, 128, 16, 50
    rotary = make_rotary(gen, d, d, total, total, 0, False)
    q, k, v = (torch.randn((total, h, d), generator=gen, device=DEV).bfloat16() for h in (H, Hk, Hk))
    m = torch.arange(total, device=DEV)
    turn = lambda x: torch.stack([turned(x[i].float(), rotary.cos[i], rotary.sin[i], False) for i in m.tolist()]).bfloat16()
    qr, kr = turn(q).double(), turn(k).double()
    want = torch.zeros((total, H, d), dtype=torch.float64, device=DEV)
    for i in range(total):
        for h in range(H):
            a = torch.softmax(kr[:i + 1, h // 2] @ qr[i, h] * d ** -0.5, 0)
            want[i, h] = a @ v[:i + 1, h // 2].double()
    for fp8, bar in ((False, OUT_RELRMS), (True, 5e-2)):
        cache = sa.alloc_cache(5, Hk, page, d, fp8=fp8)
        table = torch.tensor([[4, 1, 0, 2]], dtype=torch.int32, device=DEV)
        outs, at = [], 0
        for n in [3, 1, 1, 20, 1, 24]:
            at += n
            kv_len = torch.tensor([at], dtype=torch.int32, device=DEV)
            part = slice(at - n, at)
            rq = sa.cache_append(cache, k[part], v[part], table, kv_len, q=q[part], rotary=rotary, check_status=True)
            outs.append(sa.cache_fwd(rq, cache, table, kv_len, check_status=True))
        got = torch.cat(outs).double()
        rms = (got - want).square().mean().sqrt() / want.square().mean().sqrt()
        print(fp8, float(rms))
        assert rms <= bar


@pytest.mark.parametrize("kw", [dict(grid=(6, 11), heads=4, kv_heads=2), dict(grid=(9, 20), heads=2, kv_heads=2, fp8=False, page=128),
                                dict(grid=(1, 1), frames=70, heads=8, kv_heads=1, page=16, d=64)], ids=["frames", "bf16", "tokens"])
def test_example(kw):
    """The example's steps of streams of different ages, one of which pauses; its bound is this file's."""
    import os
    import sys
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    from examples import generate_frames
    assert generate_frames.run(**dict(dict(streams=3, frames=5, device=DEV), **kw)) <= OUT_RELRMS


# ------------------------------------------------------------------------------------- memory that threads and copies share

@pytest.mark.parametrize("fp8", [True, False])
@pytest.mark.parametrize("d,page,H,n", [(128, 64, 2, 20), (64, 16, 4, 9), (128, 32, 2, 4), (64, 128, 8, 2)])
def test_tiles_that_threads_write_between_copies(fp8, d, page, H, n):
    """Many items, nearly all of which end inside a tile and hold values that are not finite: their zeros and marks are written where the
    next item's copies go.  Every call gives the same bits, and 64-bit attention's values where nothing is broken."""
    gen = torch.Generator(device=DEV).manual_seed(d + n)
    B, Hk = 150, 2
    lens = [n + (b * 37) % 290 for b in range(B)]
    pages = sum(-(-x // page) for x in lens) + 1
    cache = make_cache(gen, pages, Hk, page, d, fp8)
    table = make_table(gen, lens, page, pages, spare=4200 // page)      # (as wide as makes a line of all items, several to a CTA)
    kv_len, q_start = batch_of(lens, [n] * B)
    q = torch.randn((B * n, H, d), generator=gen, device=DEV).bfloat16()
    kw = dict(q_start=q_start, max_new=n, return_lse=True)
    want, want_lse = reference(q[:12 * n], cache, table, lens[:12], [n] * 12, 1, 0)
    clean = sa.cache_fwd(q, cache, table, kv_len, **kw)
    check(clean[0][:12 * n], clean[1][:12 * n], want, want_lse)
    # the newest token's value is broken: the row that sees it has NaN in that channel, all others have what they had
    v = cache.v.clone(memory_format=torch.preserve_format)
    for b in range(B):
        at = (int(table[b, (lens[b] - 1) // page]), 0, (lens[b] - 1) % page, b % d)
        if fp8:
            v.view(torch.uint8)[at] = 0x7f
        else:
            v[at] = math.nan
    expected = clean[0].clone()
    for b in range(B):
        expected[(b + 1) * n - 1, :H // Hk, b % d] = math.nan
    broken = poisoned(cache._replace(v=v), table, lens, page)
    for _ in range(20):
        out, lse = sa.cache_fwd(q, broken, table, kv_len, **kw)
        assert torch.equal(torch.isnan(out), torch.isnan(expected)) and same_bits(lse, clean[1])
        assert same_bits(torch.nan_to_num(out), torch.nan_to_num(expected))


# ------------------------------------------------------------------------------------------------- zeros, and what underflows

@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 4, 8, 9, 70, 300])
@pytest.mark.parametrize("size", [0.0, 1e-5, 1e-30])
def test_rows_and_keys_of_zeros(d, n, size):
    """Queries of zeros (padding, a first step with zeroed projections) over keys of zeros, or tiny ones: every key that a row sees weighs the same,
    on both sides of the 16 rows per key head that take one kernel or the other."""
    gen = torch.Generator(device=DEV).manual_seed(n + d)
    Hk, G, page = 2, 2, 32
    lens, news = [n + 150, n], [n, n]
    k = (size * torch.randn((sum(lens), Hk, d), generator=gen, device=DEV)).bfloat16()
    v = torch.randn((sum(lens), Hk, d), generator=gen, device=DEV).bfloat16()
    for fp8 in (True, False):
        cache = sa.alloc_cache(40, Hk, page, d, fp8=fp8)
        table = make_table(gen, lens, page, 40)
        kv_len, start = batch_of(lens, lens)
        sa.cache_append(cache, k, v, table, kv_len, q_start=start, max_new=max(lens), check_status=True)
        q = torch.zeros((2 * n, Hk * G, d), dtype=torch.bfloat16, device=DEV)
        q[::3, 1] = torch.randn((len(q[::3]), d), generator=gen, device=DEV).bfloat16()      # some rows are not zeros
        _, start = batch_of(lens, news)
        for frame, window in ((1, 0), (1, 40), (7, 0), (0, 0)):
            out, lse = sa.cache_fwd(q, cache, table, kv_len, q_start=start, max_new=n, frame_tokens=frame, window=window, return_lse=True, check_status=True)
            want, want_lse = reference(q, cache, table, lens, news, frame, window)
            check(out, lse, want, want_lse)


@pytest.mark.parametrize("n", [2, 40])
def test_a_tiny_softmax_scale_is_a_mean(n):
    """A scale that all but vanishes, with masks: the mean of what a row sees."""
    gen = torch.Generator(device=DEV).manual_seed(n)
    for fp8 in (True, False):
        cache = make_cache(gen, 12, 2, 32, 128, fp8)
        lens, news = [200, 90], [n, n]
        table = make_table(gen, lens, 32, 12)
        kv_len, q_start = batch_of(lens, news)
        q = torch.randn((2 * n, 4, 128), generator=gen, device=DEV).bfloat16()
        for scale in (1e-30, 1e-44):
            out, lse = sa.cache_fwd(q, cache, table, kv_len, q_start=q_start, max_new=n, softmax_scale=scale, return_lse=True)
            want, want_lse = reference(q, cache, table, lens, news, 1, 0, scale)
            check(out, lse, want, want_lse)


def test_host_threads_with_batches_of_different_sizes():
    """Two host threads, each with a stream of its own, call the same kernel for 64 and for 1024 sequences: no call is refused, and each gives the
    bits that it gives alone."""
    import threading
    gen = torch.Generator(device=DEV).manual_seed(15)
    Hk, page, d, columns = 8, 64, 128, 80
    calls = []
    for B in (64, 1024):
        lens = [1 + i % 60 for i in range(B)]
        cache = make_cache(gen, B + 1, Hk, page, d, True)
        table = torch.zeros((B, columns), dtype=torch.int32, device=DEV)
        table[:, 0] = torch.randperm(B, generator=gen, device=DEV).int()
        kv_len, _ = batch_of(lens, [1] * B)
        q = torch.randn((B, 2 * Hk, d), generator=gen, device=DEV).bfloat16()
        want = sa.cache_fwd(q, cache, table, kv_len, check_status=True)
        calls.append((q, cache, table, kv_len, torch.empty_like(want), want, torch.empty(1 << 26, dtype=torch.uint8, device=DEV), torch.cuda.Stream()))
    torch.cuda.synchronize()
    errors = []

    def work(q, cache, table, kv_len, out, want, ws, stream):
        try:
            stream.synchronize()                                # (the thread's context is there)
            for i in range(3000):
                sa.cache_fwd(q, cache, table, kv_len, out=out, workspace=ws, stream=stream)
                if i % 100 == 99:
                    stream.synchronize()
        except Exception as e:      # (a refusal must not stay in its thread)
            errors.append(e)
    threads = [threading.Thread(target=work, args=c) for c in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors
    for c in calls:
        assert same_bits(c[4], c[5])


@pytest.mark.parametrize("n", [1, 40])
def test_a_host_threads_first_call(n):
    """A host thread whose first use of the GPU is one of these calls, with nothing left to allocate, is served as any other."""
    import threading
    gen = torch.Generator(device=DEV).manual_seed(19)
    cache = make_cache(gen, 12, 2, 64, 128, True)
    table = make_table(gen, [700], 64, 12)
    kv_len = torch.tensor([700], dtype=torch.int32, device=DEV)
    q, k = (torch.randn((n, h, 128), generator=gen, device=DEV).bfloat16() for h in (4, 2))
    want = sa.cache_fwd(q, cache, table, kv_len)
    out, ws, stream = torch.zeros_like(want), torch.empty(1 << 26, dtype=torch.uint8, device=DEV), torch.cuda.current_stream()
    dense = [torch.randn((1, 2, 512, 128), generator=gen, device=DEV).bfloat16() for _ in range(3)]
    kept, count = sa.select(*dense[:2], 128, 2)
    dense_want = sa.fwd(*dense, kept, count, 128)
    dense_out = torch.zeros_like(dense_want)
    torch.cuda.synchronize()
    calls = {"cache_fwd": lambda: sa.cache_fwd(q, cache, table, kv_len, out=out, workspace=ws, stream=stream),
             "fwd": lambda: sa.fwd(*dense, kept, count, 128, out=dense_out, workspace=ws, stream=stream),
             "cache_append": lambda: sa.cache_append(cache, k, k, table, kv_len, workspace=ws, stream=stream)}
    errors = []

    def work(name):
        try:
            calls[name]()
        except Exception as e:
            errors.append((name, e))
    for name in calls:
        thread = threading.Thread(target=work, args=(name,))
        thread.start()
        thread.join()
    torch.cuda.synchronize()
    assert not errors
    assert same_bits(out, want) and same_bits(dense_out, dense_want)


@pytest.mark.parametrize("fp8", [True, False])
@pytest.mark.parametrize("length,n", [(3000, 1), (40000, 1), (40000, 2), (40000, 30), (40000, 150)])
def test_broken_values_of_keys_far_below(fp8, length, n):
    """A value that is not finite, of a key whose logit lies 226 below the row's largest (its weight underflows), reaches every row that sees it, however
    the keys were dealt out: to one thread-block cluster, or to stretches of the line that hold nothing but such keys."""
    gen = torch.Generator(device=DEV).manual_seed(n)
    page, d, G = 64, 128, 2
    cache = make_cache(gen, -(-length // page), 1, page, d, False)
    cache.k[:] = -10.0
    first = length // 3
    table = torch.arange(-(-length // page), dtype=torch.int32, device=DEV)[None].contiguous()
    cache.k[:first // page] = 10.0
    if fp8:
        cache = sa.KVCache(*(x.to(torch.float8_e4m3fn) for x in cache[:2]), *(torch.ones((cache.k.shape[0], 1), device=DEV) for _ in range(2)))
    q = torch.ones((n, G, d), dtype=torch.bfloat16, device=DEV)
    kv_len = torch.tensor([length], dtype=torch.int32, device=DEV)
    kw = dict(max_new=n, frame_tokens=0, return_lse=True)
    clean, clean_lse = sa.cache_fwd(q, cache, table, kv_len, **kw)
    assert torch.isfinite(clean).all()
    v = cache.v.clone()
    for key, c in ((first + 100, 5), (length // 2, 77), (length - 1, 8)):
        if fp8:
            v.view(torch.uint8)[key // page, 0, key % page, c] = 0x7f
        else:
            v[key // page, 0, key % page, c] = math.nan if c != 77 else math.inf
    out, lse = sa.cache_fwd(q, cache._replace(v=v), table, kv_len, **kw)
    broken = torch.zeros(d, dtype=torch.bool, device=DEV)
    broken[[5, 77, 8]] = True
    assert (~torch.isfinite(out[..., broken])).all()
    assert same_bits(out[..., ~broken], clean[..., ~broken]) and same_bits(lse, clean_lse)


@pytest.mark.parametrize("fp8", [True, False])
@pytest.mark.parametrize("d,G,n", [(128, 1, 5), (128, 4, 4), (64, 2, 4), (64, 4, 3), (128, 4, 20), (64, 2, 150)])
def test_large_values_stay_with_who_sees_them(fp8, d, G, n):
    """Values near the type's largest among the newest tokens: the rows in front of them keep their bits, and where all that a row sees is zero, so is
    its output."""
    gen = torch.Generator(device=DEV).manual_seed(n + G)
    page, Hk, length = 32, 2, 100 + n
    cache = make_cache(gen, 12, Hk, page, d, fp8)
    table = make_table(gen, [length], page, 12)
    kv_len = torch.tensor([length], dtype=torch.int32, device=DEV)
    q = torch.randn((n, Hk * G, d), generator=gen, device=DEV).bfloat16()
    kw = dict(max_new=n, return_lse=True)
    seen = length - n + n // 2                                  # keys of the rows in front of row n // 2
    for zeros, large in ((False, 1e30), (True, 1e30), (False, 3e38), (True, 3e38)):
        v = cache.v.clone(memory_format=torch.preserve_format)
        bits = v.view(torch.uint8) if fp8 else v
        if zeros:
            bits.zero_()
        clean, clean_lse = sa.cache_fwd(q, cache._replace(v=v), table, kv_len, **kw)
        for j in range(seen, length):
            bits[int(table[0, j // page]), :, j % page] = 0x7e if fp8 else large
        out, lse = sa.cache_fwd(q, cache._replace(v=v), table, kv_len, **kw)
        assert same_bits(lse, clean_lse)
        assert same_bits(out[:n // 2], clean[:n // 2])
        assert not zeros or (out[:n // 2] == 0).all()
        if large == 3e38:                                       # (sums of weights up to 2^15 times such values pass fp32)
            continue
        want, _ = reference(q, cache._replace(v=v), table, [length], [n], 1, 0)
        assert ((out.double() - want).abs() <= OUT_MAX_OF_ROW * want.abs().amax(-1, keepdim=True)).all()


@pytest.mark.parametrize("n", [1, 2, 30])
def test_small_weights_of_large_values(n):
    """bf16 pages: a key of weight 2^-120 with values of 2^126 beside one of weight 1 with values of 1."""
    page, d = 16, 128
    cache = sa.alloc_cache(2, 1, page, d, fp8=False)
    cache.k[0, 0, 0] = 0.0
    cache.k[0, 0, 1] = -120 * math.log(2.0) / math.sqrt(d)
    cache.v[0, 0, 0], cache.v[0, 0, 1] = 1.0, 2.0 ** 126
    q = torch.ones((n, 1, d), dtype=torch.bfloat16, device=DEV)
    table = torch.zeros((1, 1), dtype=torch.int32, device=DEV)
    kv_len = torch.tensor([2], dtype=torch.int32, device=DEV)
    if n > 2:
        kv_len += n - 2
        cache.k[0, 0, 2:] = cache.k[0, 0, 1]
        cache.k[1, 0] = cache.k[0, 0, 1]
        table = torch.tensor([[0, 1]], dtype=torch.int32, device=DEV)
    lens = [int(kv_len)]
    out = sa.cache_fwd(q, cache, table, kv_len, max_new=n, frame_tokens=0, check_status=True)
    want, _ = reference(q, cache, table, lens, [n], 0, 0)
    # (the logit's own rounding: 2^-23 of 83, times the exponential)
    assert ((out.double() - want).abs() <= OUT_MAX_OF_ROW * want.abs().amax(-1, keepdim=True)).all()


@pytest.mark.parametrize("frame,n", [(1, 1), (50, 3), (7, 30)])
def test_a_window_of_any_size(frame, n):
    """The widest window that an int holds is no window: the same keys, dealt out in the same way, the same bits."""
    gen = torch.Generator(device=DEV).manual_seed(frame)
    lens, news = [3001, 700], [n, n]
    cache = make_cache(gen, 60, 2, 64, 128, True)
    table = make_table(gen, lens, 64, 60, spare=0)
    kv_len, q_start = batch_of(lens, news)
    q = torch.randn((2 * n, 4, 128), generator=gen, device=DEV).bfloat16()
    want, want_lse = sa.cache_fwd(q, cache, table, kv_len, max_new=n, frame_tokens=frame, return_lse=True)
    for window in (2 ** 31 - 1, 2 ** 31 - 2, 10 ** 6):
        out, lse = sa.cache_fwd(q, cache, table, kv_len, max_new=n, frame_tokens=frame, window=window, return_lse=True, check_status=True)
        assert same_bits(out, want) and same_bits(lse, want_lse)


def test_memory_of_calls_on_another_stream():
    """What a call allocates itself for a stream of the caller's is neither memory that the current stream may still use, nor handed out to the
    current stream while the other has yet to use it."""
    gen = torch.Generator(device=DEV).manual_seed(17)
    cache = make_cache(gen, 40, 2, 64, 128, True)
    table = make_table(gen, [2000], 64, 40)
    kv_len = torch.tensor([2000], dtype=torch.int32, device=DEV)
    q = torch.randn((1, 4, 128), generator=gen, device=DEV).bfloat16()
    k = torch.randn((1, 2, 128), generator=gen, device=DEV).bfloat16()
    x = torch.randn((1, 2, 512, 128), generator=gen, device=DEV).bfloat16()
    kept, count = sa.select(x, x, 128, 2)
    index = torch.arange(512, device=DEV, dtype=torch.int32)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    to, native = side.cuda_stream, sa._calls()
    calls = {"cache_fwd": lambda: native.cache_fwd(*cache, table, kv_len, None, 0, q, 1, 0, 0.0, None, True, None, to),
             "cache_append": lambda: native.cache_append(*cache, table, kv_len, None, 0, k, k, q, None, None, None, None, None, False, None, to),
             "select": lambda: native.select(x, x, 128, 2, None, None, None, to, 0, 0, None),
             "quant_fp8": lambda: native.quant_fp8(x, 128, None, None, to),
             "fwd": lambda: native.fwd(x, x, x, kept, count, 128, sa.BF16, None, None, None, 0.0, None, True, None, to, 0, 0, None),
             "gather_tokens": lambda: native.gather_tokens(x, index, None, None, to)}
    places = lambda tensors: [(y.data_ptr(), y.data_ptr() + y.numel() * y.element_size()) for y in tensors if y is not None]
    apart = lambda a, b: all(hi <= x0 or x1 <= lo for lo, hi in a for x0, x1 in b)
    for name, call in calls.items():
        rc, *made = call()
        assert rc == sa.OK
        sizes = [hi - lo for lo, hi in places(made)]
        del made
        torch.cuda.synchronize()
        # memory that the current stream has given back, and may still be working on
        freed = [torch.empty(size, dtype=torch.uint8, device=DEV) for size in sizes for _ in range(4)]
        torch.cuda._sleep(20_000_000)
        used = places(freed)
        del freed
        rc, *made = call()
        assert apart(places(made), used), name
        torch.cuda.synchronize()
        # the other stream has not begun when what the call made is dropped
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)
        rc, *made = call()
        used = places(made)
        del made
        others = [torch.empty(size, dtype=torch.uint8, device=DEV) for size in sizes for _ in range(4)]
        assert apart(places(others), used), name
        torch.cuda.synchronize()
        # an output that the current stream reads is not overwritten by the other's next call
        rc, *made = call()
        out = places(made[:1])
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda._sleep(200_000_000)                          # (0.1 s: the host is back in time)
        del made
        rc, *made = call()
        assert apart(places(made), out), name
        torch.cuda.synchronize()


# ------------------------------------------------------------------------------------------------------ inside the tensors

def margined(x):
    """x's bits as a view into a larger buffer, and the buffer: one of a known byte, on both sides, and between rows of the last dimension but two."""
    outer = list(x.shape)
    outer[0] += 2                                               # a whole block in front and behind
    if x.dim() > 2:
        outer[-2] += 1                                          # and a row behind each block's rows
    buf = torch.empty(outer, dtype=x.dtype, device=DEV)
    buf.view(torch.uint8).fill_(0xA5)
    inner = buf[1:-1, ..., :-1, :] if x.dim() > 2 else buf[1:-1]
    inner.copy_(x)
    return inner, buf


def margins_kept(inner, buf):
    bits = buf.view(torch.uint8).clone()
    same = torch.full_like(bits, 0xA5)
    inside = (lambda x: x[1:-1, ..., :-1, :]) if buf.dim() > 2 else (lambda x: x[1:-1])
    inside(bits).copy_(inside(same))
    return torch.equal(bits, same)


@pytest.mark.parametrize("what", ["nothing", "negative length", "length beyond the table", "starts descend", "starts beyond the rows", "more than max_new",
                                  "more new tokens than tokens", "pages that do not exist"])
@pytest.mark.parametrize("fp8,G", [(True, 2), (False, 2), (True, 9), (False, 9)])
def test_a_broken_callers_numbers_touch_nothing_else(what, fp8, G):
    """Pools, scales, rows and outputs inside larger buffers: whatever the device-side numbers are, the margins, pages of nobody and the tokens in front of
    the new ones keep their bits."""
    gen = torch.Generator(device=DEV).manual_seed(16)
    Hk, page, d, n = 2, 16, 64, 3
    cache = make_cache(gen, 9, Hk, page, d, fp8)
    held = [None if x is None else margined(x) for x in cache]
    cache = sa.KVCache(*(None if x is None else x[0] for x in held))
    if cache.k_scale is not None:                               # (scales are contiguous: rows in front and behind)
        assert cache.k_scale.is_contiguous()
    lens, starts = [40, 50], [0, 3, 6]
    table = make_table(gen, lens, page, 9, spare=0)
    table[0, 3] = table[0, 0]                                   # (a column that a length of 40 does not reach)
    owned = {b: set(table[b, :-(-x // page)].tolist()) for b, x in enumerate(lens)}
    max_new = n
    if what == "negative length":
        lens[0] = -5
    elif what == "length beyond the table":
        lens[1] = 100000
    elif what == "starts descend":
        starts = [4, 2, 6]
    elif what == "starts beyond the rows":
        starts = [0, 3, 900]
    elif what == "more than max_new":
        max_new = 2
    elif what == "more new tokens than tokens":
        lens[0] = 2
    elif what == "pages that do not exist":
        table[0, 2], table[1, 1] = 9, -1
    kv_len = torch.tensor(lens, dtype=torch.int32, device=DEV)
    q_start = torch.tensor(starts, dtype=torch.int32, device=DEV)
    q = torch.randn((6, Hk * G, d), generator=gen, device=DEV).bfloat16()
    k, v = (torch.randn((6, Hk, d), generator=gen, device=DEV).bfloat16() for _ in range(2))
    outs = [margined(torch.zeros_like(q)) for _ in range(2)]
    ws = torch.empty(1 << 26, dtype=torch.uint8, device=DEV)
    before = [None if x is None else x.clone() for x in cache]
    status = sa.OK if what == "nothing" else sa.E_BAD_INDEX
    sa.cache_fwd(q, cache, table, kv_len, q_start=q_start, max_new=max_new, out=outs[0][0], workspace=ws)
    assert sa.read_status(ws) == status
    for x, y in zip(cache, before):
        assert x is None or same_bits(x, y)                     # (it reads)
    sa.cache_append(cache, k, v, table, kv_len, q_start=q_start, max_new=max_new, q=q, q_out=outs[1][0], workspace=ws)
    assert sa.read_status(ws) == status
    for x in (*held, *outs):
        assert x is None or margins_kept(*x)
    nobodys = [p for p in range(9) if p not in owned[0] | owned[1]]
    for x, y in zip(cache, before):
        assert x is None or same_bits(x[nobodys], y[nobodys])
    # pages that a sequence has filled before: all but the one where its new tokens begin, where the numbers are its own
    for b, first in ((0, 37 // page), (1, 47 // page)):
        if what in ("nothing", "more than max_new", "pages that do not exist"):
            full = [p for p in table[b, :first].tolist() if 0 <= p < 9]
            for x, y in zip(cache, before):
                assert x is None or same_bits(x[full], y[full])


# ------------------------------------------------------------------------------------- forms that the cases above leave out

@pytest.mark.parametrize("case", [
    ([1000, 130], [10, 9], 16, 4, 128, 64, False, 1, 0),       # 40 rows of 128 channels, bf16
    ([700], [100], 1, 1, 128, 16, False, 1, 90),
    ([3000, 20], [16, 3], 8, 1, 128, 128, False, 30, 2),
    ([500, 0, 300], [16, 2, 16], 8, 8, 128, 32, False, 1, 0),  # 16 rows, one group of keys a warp
    ([600], [8], 8, 4, 64, 32, False, 1, 0),
    ([1, 4000, 17], [1, 500, 1], 4, 2, 64, 16, True, 1, 0),    # a prompt's piece beside single tokens
    ([1, 900, 17], [1, 300, 1], 8, 8, 128, 64, False, 1, 0),
], ids=lambda c: "-".join(str(x) for x in c[2:]) + f"-{len(c[0])}x{max(c[0])}")
def test_attention_over_pages_of_other_forms(case):
    test_attention_over_pages(case, False)


@pytest.mark.parametrize("fp8", [True, False])
@pytest.mark.parametrize("n", [1, 2, 30])
def test_a_table_wider_than_the_lengths(fp8, n):
    """A serving loop's table has columns for the longest context allowed: the result is attention's, whatever the width."""
    gen = torch.Generator(device=DEV).manual_seed(18)
    lens, news = [1000, 77], [n, n]
    cache = make_cache(gen, 40, 2, 32, 128, fp8)
    kv_len, q_start = batch_of(lens, news)
    q = torch.randn((2 * n, 16, 128), generator=gen, device=DEV).bfloat16()
    table = make_table(gen, lens, 32, 40)
    want, want_lse = reference(q, cache, table, lens, news, 1, 0)
    for columns in (32, 128, 1000, 4096):
        wide = torch.full((2, columns), -7, dtype=torch.int32, device=DEV)
        wide[:, :32] = table[:, :32]
        out, lse = sa.cache_fwd(q, cache, wide, kv_len, q_start=q_start, max_new=n, return_lse=True, check_status=True)
        check(out, lse, want, want_lse)


@pytest.mark.parametrize("n", [1, 30])
def test_scales_of_any_size(n):
    """Scales of a page and head anywhere from 2^-64 to 2^60, side by side; a value scale below 2^-64 counts as that."""
    gen = torch.Generator(device=DEV).manual_seed(20)
    lens, page, d = [300], 32, 64
    cache = make_cache(gen, 12, 2, page, d, True)
    table = make_table(gen, lens, page, 12)
    kv_len = torch.tensor(lens, dtype=torch.int32, device=DEV)
    q = torch.randn((n, 4, d), generator=gen, device=DEV).bfloat16()
    for low, high in ((-64, -60), (-8, 60), (-64, 0), (20, 60)):
        scale = torch.exp2(torch.randint(low, high + 1, (12, 2), generator=gen, device=DEV).float())
        c = cache._replace(v_scale=scale)
        out, lse = sa.cache_fwd(q, c, table, kv_len, max_new=n, return_lse=True, check_status=True)
        want, want_lse = reference(q, c, table, lens, [n], 1, 0)
        size = want.abs().amax(-1, keepdim=True)
        assert ((out.double() - want).abs() <= OUT_MAX_OF_ROW * size).all() and (lse - want_lse).abs().max() <= LSE_ABS
    tiny = sa.cache_fwd(q, cache._replace(v_scale=torch.full_like(scale, 2.0 ** -100)), table, kv_len, max_new=n)
    least = sa.cache_fwd(q, cache._replace(v_scale=torch.full_like(scale, 2.0 ** -64)), table, kv_len, max_new=n)
    assert same_bits(tiny, least)
