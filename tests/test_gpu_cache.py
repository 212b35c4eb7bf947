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
