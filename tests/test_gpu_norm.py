"""GPU parity of the norm of queries and keys with their rotation, over whole sequences and on the way into a paged cache, against the formula
in 64 bits.

Bounds: the result is rounded to bf16 once, 2^-8 of it at most.  Before that every channel has passed a sum of squares (127 additions at most,
but in a tree: relative 2^-24 times about 12, halved by the root), the root (2 units of 2^-23 by CUDA's documentation), two products and the
rotation's three roundings: below 2^-19 of the sum of the magnitudes that the rotation adds up."""
import math

import pytest
import torch

import paper_2609_23153_b200 as sa
from test_gpu_cache import DEV, append_reference, batch_of, make_cache, make_rotary, make_table, same_bits

pytestmark = pytest.mark.gpu
ROUNDING, BEFORE = 2.0 ** -8, 2.0 ** -19


def normed64(x, weight, eps):
    x = x.double()
    y = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
    return y if weight is None else y * weight.double()


def turned64(x, rotary, pos):
    """(x [..., T, d] turned, the magnitudes that were added up)"""
    if rotary is None:
        return x, x.abs()
    cos, sin, positions, axis, inter = rotary
    pairs = cos.shape[1]
    m = torch.arange(pairs, device=x.device)
    at = pos[:, None].expand(-1, pairs) if positions is None else positions.view(len(positions), -1).long()[:, torch.zeros_like(m) if axis is None else axis.long()]
    c, s = cos[at, m].double(), sin[at, m].double()
    a, b = (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)) if inter else (slice(0, pairs), slice(pairs, 2 * pairs))
    y, size = x.clone(), x.abs()
    p, q = x[..., a], x[..., b]
    y[..., a], y[..., b] = p * c - q * s, p * s + q * c
    size[..., a], size[..., b] = (p * c).abs() + (q * s).abs(), (p * s).abs() + (q * c).abs()
    return y, size


def near(got, want, size, step=ROUNDING):
    off = (got.double() - want).abs()
    assert (off <= step * want.abs() + BEFORE * size).all(), float((off - step * want.abs() - BEFORE * size).max())


def weights(gen, H, d, dtype, per_head):
    if dtype is None:
        return None
    return (1 + 0.5 * torch.randn((H, d) if per_head else (d,), generator=gen, device=DEV)).to(dtype)


def tensors(gen, B, H, Hk, N, d, layout):
    x = torch.randn((B, N, H + 2 * Hk, d), generator=gen, device=DEV) * torch.exp(2 * torch.randn((B, N, H + 2 * Hk, 1), generator=gen, device=DEV))
    x = x.bfloat16()
    if layout == "qkv":        # parts of a fused projection's rows
        y = x.transpose(1, 2)
        return y[:, :H], y[:, H:H + Hk]
    q, k = x[:, :, :H].transpose(1, 2), x[:, :, H:H + Hk].transpose(1, 2)
    return (q.contiguous(), k.contiguous()) if layout == "bhnd" else (q.transpose(1, 2).contiguous().transpose(1, 2), k.contiguous())


WHOLE = [
    # B, H, Hk, N, d, rot, axes, interleaved, weight, per_head, layout
    (1, 1, 1, 1, 128, 128, 0, False, torch.float32, False, "bhnd"),
    (1, 3, 1, 17, 128, 128, 3, True, torch.bfloat16, False, "qkv"),
    (2, 6, 2, 1201, 64, 32, 0, False, torch.bfloat16, True, "bnhd"),
    (3, 5, 5, 333, 64, 64, 2, True, torch.float32, True, "qkv"),
    (1, 12, 12, 4097, 128, 64, 1, False, None, False, "bhnd"),
    (2, 40, 8, 65, 128, 16, 0, True, torch.float32, True, "bnhd"),
    (1, 2, 2, 20000, 128, 128, 3, True, torch.float32, False, "bnhd"),
    (1, 7, 3, 50, 64, 0, 0, False, torch.float32, False, "qkv"),
    (4, 64, 1, 9, 64, 16, 4, False, torch.bfloat16, True, "qkv"),
]


@pytest.mark.parametrize("case", WHOLE, ids=lambda c: "-".join(str(x) for x in c))
@pytest.mark.parametrize("eps", [1e-6, 0.5])
def test_whole_sequences(case, eps):
    B, H, Hk, N, d, rot, axes, inter, dtype, per_head, layout = case
    gen = torch.Generator(device=DEV).manual_seed(N + H)
    q, k = tensors(gen, B, H, Hk, N, d, layout)
    q[0, 0, N // 2], k[-1, -1, N - 1] = 0.0, 0.0
    rotary = make_rotary(gen, d, rot, max(N, 70), N, axes, inter) if rot else None
    norm = sa.Norm(weights(gen, H, d, dtype, per_head), weights(gen, Hk, d, dtype, per_head), eps)
    ws = torch.full((256,), 0xA5, dtype=torch.uint8, device=DEV)
    got = sa.norm_rotate(q, k, norm=norm, rotary=rotary, workspace=ws)
    assert sa.read_status(ws) == sa.OK
    pos = torch.arange(N, device=DEV)
    for x, y, w in ((q, got[0], norm.q), (k, got[1], norm.k)):
        assert y.shape == x.shape and y.stride() == x.stride()
        want, size = turned64(normed64(x, w[:, None] if w is not None and per_head else w, eps), rotary, pos)
        near(y, want, size)
    assert (got[0][0, 0, N // 2] == 0).all() and (got[1][-1, -1, N - 1] == 0).all()
    # queries alone, and in place: the same bits
    assert same_bits(sa.norm_rotate(q, norm=norm, rotary=rotary), got[0])
    want = [x.clone() for x in got]
    there = sa.norm_rotate(q, k, norm=norm, rotary=rotary, q_out=q, k_out=k)
    assert all(a.data_ptr() == b.data_ptr() and same_bits(a, c) for a, b, c in zip(there, (q, k), want))


def test_rotation_alone_has_the_bits_of_the_cache():
    gen = torch.Generator(device=DEV).manual_seed(1)
    for d, rot, axes, inter in ((128, 128, 0, False), (128, 64, 3, True), (64, 64, 2, False), (64, 16, 0, True)):
        N, H = 130, 3
        x = torch.randn((1, H, N, d), generator=gen, device=DEV).bfloat16()
        rotary = make_rotary(gen, d, rot, N, N, axes, inter)
        got = sa.norm_rotate(x, rotary=rotary, check_status=True)
        cache = sa.alloc_cache(4, H, 64, d, fp8=False, device=DEV)
        table, kv_len = torch.arange(4, dtype=torch.int32, device=DEV)[None].contiguous(), torch.tensor([N], dtype=torch.int32, device=DEV)
        rows = x[0].transpose(0, 1)
        sa.cache_append(cache, rows, rows, table, kv_len, rotary=rotary, check_status=True)
        stored = cache.k.transpose(0, 1).reshape(H, -1, d)[:, :N]
        assert same_bits(got[0], stored)


def test_rows_around_the_output_stay():
    gen = torch.Generator(device=DEV).manual_seed(2)
    for d in (64, 128):
        x = torch.randn((2, 3, 37, d), generator=gen, device=DEV).bfloat16()
        room = torch.full((4, 5, 60, d), 7.0, device=DEV).bfloat16()
        out = room[1:3, 1:4, 11:48]
        sa.norm_rotate(x, norm=sa.Norm(), q_out=out)
        near(out, normed64(x, None, 1e-6), normed64(x, None, 1e-6).abs())
        out.fill_(7.0)
        assert (room == 7.0).all()


def test_broken_rows_stay_alone():
    """An infinity or a NaN breaks its row, the largest numbers (whose squares pass fp32's range) give zeros, and the other rows keep their bits."""
    gen = torch.Generator(device=DEV).manual_seed(3)
    x = torch.randn((1, 2, 40, 128), generator=gen, device=DEV).bfloat16()
    norm = sa.Norm()
    clean = sa.norm_rotate(x, norm=norm)
    y = x.clone()
    y[0, 0, 3, 7], y[0, 0, 4, 100], y[0, 1, 5] = math.inf, math.nan, 2e38
    y[0, 1, 6] = 1e-30
    got = sa.norm_rotate(y, norm=norm)
    assert torch.isnan(got[0, 0, 3, 7]) and (got[0, 0, 3, :7] == 0).all() and torch.isnan(got[0, 0, 4]).all() and (got[0, 1, 5] == 0).all()
    near(got[0, 1, 6], normed64(y[0, 1, 6], None, 1e-6), normed64(y[0, 1, 6], None, 1e-6).abs())
    same = torch.ones(40, dtype=torch.bool, device=DEV)
    same[3:7] = False
    assert same_bits(got[:, :, same], clean[:, :, same])


@pytest.mark.parametrize("word", [0, -7, -6, 0x5A5A5A5A])
def test_positions_outside_the_tables(word):
    gen = torch.Generator(device=DEV).manual_seed(4)
    N = 900
    x = torch.randn((1, 2, N, 128), generator=gen, device=DEV).bfloat16()
    ws = torch.zeros(64, dtype=torch.int32, device=DEV)

    def status(rotary):
        ws[0] = word
        out = sa.norm_rotate(x, norm=sa.Norm(), rotary=rotary, workspace=ws.view(torch.uint8))
        return sa.read_status(ws.view(torch.uint8)), out

    rotary = make_rotary(gen, 128, 64, 50, N, 2, True)
    plain = sa.norm_rotate(x, norm=sa.Norm())
    good, want = status(rotary)
    assert good == sa.OK
    bad = rotary.positions.clone()
    bad[777, 0] = 50
    bad[800, 1] = -1
    code, got = status(rotary._replace(positions=bad))
    assert code == sa.E_BAD_INDEX
    m = torch.arange(32, device=DEV)
    for t, ax in ((777, 0), (800, 1)):
        left = (rotary.axis == ax).repeat_interleave(2)                    # these pairs are not turned
        assert same_bits(got[0, :, t, :64][:, left], plain[0, :, t, :64][:, left])
        assert same_bits(got[0, :, t, :64][:, ~left], want[0, :, t, :64][:, ~left])
    axis = rotary.axis.clone()
    axis[5] = 2
    assert status(rotary._replace(axis=axis))[0] == sa.E_BAD_INDEX
    short = make_rotary(gen, 128, 128, N - 1, N, 0, False)
    assert status(short)[0] == sa.E_BAD_INDEX
    assert status(make_rotary(gen, 128, 128, N, N, 0, False))[0] == sa.OK


APPENDS = [
    # lens, news, H, Hk, d, page, fp8, rot, axes, interleaved, weight, per_head
    ([1], [1], 8, 8, 128, 16, False, 128, 0, False, torch.float32, False),
    ([64, 65, 190], [1, 1, 1], 40, 8, 128, 64, True, 64, 0, False, torch.bfloat16, False),
    ([5, 17, 33, 64], [5, 3, 16, 1], 6, 2, 64, 16, True, 64, 0, True, torch.float32, True),
    ([300, 130], [300, 129], 4, 4, 128, 128, True, 128, 3, True, torch.bfloat16, True),
    ([300, 130], [290, 130], 3, 1, 128, 64, False, 32, 0, False, torch.float32, True),
    ([77], [70], 2, 2, 64, 32, False, 64, 2, False, None, False),
    ([200, 9, 1], [100, 2, 1], 5, 5, 64, 128, True, 16, 0, False, torch.float32, False),
    ([200, 90], [37, 33], 16, 4, 128, 32, True, 0, 0, False, torch.bfloat16, False),
    ([1000, 40], [2, 4], 8, 1, 128, 128, False, 128, 1, False, torch.float32, True),
]


@pytest.mark.parametrize("case", APPENDS, ids=lambda c: "-".join(str(x) for x in c[2:]) + f"-{len(c[0])}x{max(c[1])}")
@pytest.mark.parametrize("layout", ["hnd", "nhd"])
def test_append(case, layout):
    """Queries and bf16 pages have the bits of norm_rotate; E4M3 pages hold the formula's values to half a step of their codes; values and whatever
    was there go their way as without the norm."""
    lens, news, H, Hk, d, page, fp8, rot, axes, inter, dtype, per_head = case
    gen = torch.Generator(device=DEV).manual_seed(sum(lens) + d)
    pages = sum(-(-n // page) for n in lens) + 2
    cache = make_cache(gen, pages, Hk, page, d, fp8, layout=layout)
    table = make_table(gen, lens, page, pages)
    kv_len, q_start = batch_of(lens, news)
    T = sum(news)
    qkv = (torch.randn((T, H + 2 * Hk, d), generator=gen, device=DEV) * torch.exp(1.5 * torch.randn((T, 1, 1), generator=gen, device=DEV))).bfloat16()
    q, k, v = qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:]
    pos = torch.cat([torch.arange(n - m, n, device=DEV) for n, m in zip(lens, news)])
    rotary = make_rotary(gen, d, rot, max(lens), T, axes, inter) if rot else None
    norm = sa.Norm(weights(gen, H, d, dtype, per_head), weights(gen, Hk, d, dtype, per_head))
    before = sa.KVCache(*(None if x is None else x.clone() for x in cache))
    plain, _ = append_reference(before, k, v, table, lens, news, None, None)          # what becomes of values, and of rows that were there
    ws = torch.full((256,), 0xA5, dtype=torch.uint8, device=DEV)
    got_q = sa.cache_append(cache, k, v, table, kv_len, q_start=q_start, max_new=max(news), q=q, norm=norm, rotary=rotary, workspace=ws)
    assert sa.read_status(ws) == sa.OK
    assert same_bits(cache.v, plain.v) and (not fp8 or same_bits(cache.v_scale, plain.v_scale))
    here = None if rotary is None else rotary._replace(positions=pos.int() if rotary.positions is None else rotary.positions,
                                                       axis=None if rotary.positions is None else rotary.axis)
    one_q, one_k = sa.norm_rotate(q.transpose(0, 1)[None], k.transpose(0, 1)[None], norm=norm, rotary=here, check_status=True)
    assert same_bits(got_q, one_q[0].transpose(0, 1))
    t = 0
    for b, (length, n) in enumerate(zip(lens, news)):
        at = torch.arange(length - n, length, device=DEV)
        pg, slot = table[b, at // page].long(), at % page
        if not fp8:
            assert same_bits(cache.k[pg, :, slot], one_k[0].transpose(0, 1)[t:t + n])
        else:
            w = norm.k if norm.k is None or not per_head else norm.k[:, None]
            part = None if here is None else here._replace(positions=here.positions[t:t + n])
            want, size = turned64(normed64(k[t:t + n].transpose(0, 1), w, 1e-6), part, at)
            scale = cache.k_scale[pg].double()[..., None]
            assert (torch.frexp(cache.k_scale)[0] == 0.5).all()
            off = (cache.k[pg, :, slot].double() * scale - want.transpose(0, 1)).abs()
            assert (off <= 2.0 ** -4 * want.transpose(0, 1).abs() + 2.0 ** -10 * scale + BEFORE * size.transpose(0, 1)).all()
            # no value is clipped, and no page's scale is twice what it needs (one that held tokens keeps what they needed)
            assert (want.transpose(0, 1).abs() <= 448 * scale * (1 + 2.0 ** -4)).all()
            for i in range((length - n) // page, -(-length // page)):
                mine = (at // page) == i
                top = want[:, mine].abs().amax(dim=(1, 2))
                kept = before.k_scale[table[b, i]].double() if i * page < length - n else torch.zeros_like(top)
                assert (cache.k_scale[table[b, i]].double() / 2 * 448 * (1 - 1e-6) <= torch.maximum(top, kept * 224 * 2)).all()
        t += n
    again = sa.cache_append(cache, k, v, table, kv_len, q_start=q_start, max_new=max(news), q=q, q_out=q, norm=norm, rotary=rotary)
    assert again.data_ptr() == q.data_ptr() and same_bits(again, got_q)


@pytest.mark.parametrize("fp8", [True, False])
def test_pieces_and_all_at_once(fp8):
    """A bf16 page holds the same bits however its tokens came; so do the queries."""
    gen = torch.Generator(device=DEV).manual_seed(8)
    T, H, d, page = 150, 2, 128, 32
    q, k, v = (torch.randn((T, H, d), generator=gen, device=DEV).bfloat16() for _ in range(3))
    rotary = make_rotary(gen, d, 64, T, T, 0, True)
    norm = sa.Norm(weights(gen, H, d, torch.float32, False), weights(gen, H, d, torch.float32, False))
    table = torch.arange(5, dtype=torch.int32, device=DEV)[None].contiguous()
    whole, parts = (sa.alloc_cache(5, H, page, d, fp8=fp8, device=DEV) for _ in range(2))
    one = sa.cache_append(whole, k, v, table, torch.tensor([T], dtype=torch.int32, device=DEV), q=q, norm=norm, rotary=rotary, check_status=True)
    got, at = [], 0
    for n in (1, 1, 3, 27, 40, 7, 64, 7):
        at += n
        got.append(sa.cache_append(parts, k[at - n:at], v[at - n:at], table, torch.tensor([at], dtype=torch.int32, device=DEV), q=q[at - n:at], norm=norm,
                                   rotary=rotary, check_status=True))
    assert at == T and same_bits(torch.cat(got), one)
    if not fp8:
        assert same_bits(whole.k, parts.k) and same_bits(whole.v, parts.v)
    else:
        assert same_bits(whole.k_scale, parts.k_scale)


def test_captured_and_on_another_stream():
    gen = torch.Generator(device=DEV).manual_seed(9)
    q, k = (torch.randn((2, 4, 500, 128), generator=gen, device=DEV).bfloat16() for _ in range(2))
    rotary = make_rotary(gen, 128, 128, 500, 500, 0, False)
    norm = sa.Norm(weights(gen, 4, 128, torch.float32, False), None)
    want = sa.norm_rotate(q, k, norm=norm, rotary=rotary)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = sa.norm_rotate(q, k, norm=norm, rotary=rotary, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(same_bits(a, b) for a, b in zip(got, want))
    outs = [torch.empty_like(q) for _ in range(2)]
    ws = torch.empty(256, dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sa.norm_rotate(q, k, norm=norm, rotary=rotary, q_out=outs[0], k_out=outs[1], workspace=ws)
    q.copy_(torch.randn(q.shape, generator=gen, device=DEV))
    graph.replay()
    again = sa.norm_rotate(q, k, norm=norm, rotary=rotary)
    assert all(same_bits(a, b) for a, b in zip(outs, again)) and not same_bits(again[0], want[0])


def test_more_than_2_to_the_32_bytes():
    """Rows far apart: a sequence whose heads together pass 2^32 bytes."""
    gen = torch.Generator(device=DEV).manual_seed(10)
    N, H = 300000, 60
    q = torch.empty((1, H, N, 128), dtype=torch.bfloat16, device=DEV)
    assert q.numel() * 2 > 2 ** 32
    for h in range(H):
        q[0, h] = torch.randn((N, 128), generator=gen, device=DEV, dtype=torch.bfloat16)
    rotary = make_rotary(gen, 128, 128, N, N, 0, True)
    want = {}
    for h, n in ((0, 0), (0, N - 1), (H // 2, N // 2), (H - 1, 0), (H - 1, N - 1)):
        want[h, n] = turned64(normed64(q[0, h, n:n + 1], None, 1e-6), rotary, torch.tensor([n], device=DEV))
    sa.norm_rotate(q, norm=sa.Norm(), rotary=rotary, q_out=q, check_status=True)
    for (h, n), (x, size) in want.items():
        near(q[0, h, n:n + 1], x, size)


def test_attention_and_norm_over_odd_strides():
    """Heads of a larger tensor, every second token, both samples of a batch in one storage."""
    gen = torch.Generator(device=DEV).manual_seed(11)
    big = torch.randn((2, 90, 7, 192), generator=gen, device=DEV).bfloat16()
    x = big[:, ::2, 1:6, 64:].transpose(1, 2)
    assert x.shape == (2, 5, 45, 128) and x.stride(3) == 1
    got = sa.norm_rotate(x, norm=sa.Norm(), check_status=True)
    near(got, normed64(x, None, 1e-6), normed64(x, None, 1e-6).abs())


@pytest.mark.parametrize("word", [0, -7])
def test_positions_of_many_tokens(word):
    """What stands in the positions of an axis that no pair turns by is not looked at, and one number among many is found whatever the
    workspace held."""
    gen = torch.Generator(device=DEV).manual_seed(14)
    N = 70001
    x = torch.randn((1, 1, N, 64), generator=gen, device=DEV).bfloat16()
    ws = torch.zeros(64, dtype=torch.int32, device=DEV)
    rotary = make_rotary(gen, 64, 64, 50, N, 3, True)
    positions, axis = rotary.positions.clone(), torch.where(rotary.axis == 1, 2, rotary.axis).int()
    positions[:, 1] = 1000
    want = sa.norm_rotate(x, norm=sa.Norm(), rotary=rotary._replace(axis=axis))
    for token, ax, code in ((0, 1, sa.OK), (N - 1, 2, sa.E_BAD_INDEX), (12345, 0, sa.E_BAD_INDEX)):
        bad = positions.clone()
        bad[token, ax] = -5
        ws[0] = word
        got = sa.norm_rotate(x, norm=sa.Norm(), rotary=rotary._replace(positions=bad, axis=axis), workspace=ws.view(torch.uint8))
        assert sa.read_status(ws.view(torch.uint8)) == code
        rest = torch.arange(N, device=DEV) != token
        assert same_bits(got[:, :, rest], want[:, :, rest])


@pytest.mark.parametrize("shift", range(4))
@pytest.mark.parametrize("T", [1, 3, 700, 4999])
def test_positions_that_begin_anywhere(shift, T):
    """Positions whose first number lies 4, 8 or 12 bytes behind a 16-byte boundary: a bad one is reported wherever it stands."""
    gen = torch.Generator(device=DEV).manual_seed(T)
    cache = sa.alloc_cache(-(-T // 64), 1, 64, 64, fp8=True, device=DEV)
    k = torch.randn((T, 1, 64), generator=gen, device=DEV).bfloat16()
    table = torch.arange(cache.k.shape[0], dtype=torch.int32, device=DEV)[None]
    kv_len = torch.tensor([T], dtype=torch.int32, device=DEV)
    rotary = make_rotary(gen, 64, 64, 50, T, 3, True)
    whole = torch.full((shift + 3 * T + 8,), -1, dtype=torch.int32, device=DEV)           # (what lies around them is not looked at)
    positions = whole[shift:shift + 3 * T].view(T, 3)
    positions.copy_(rotary.positions)
    ws = torch.empty(256, dtype=torch.uint8, device=DEV)
    sa.cache_append(cache, k, k, table, kv_len, rotary=rotary._replace(positions=positions), workspace=ws)
    assert sa.read_status(ws) == sa.OK
    for at in sorted({0, 1, 3 * T // 2, 3 * T - 2, 3 * T - 1}):
        positions.copy_(rotary.positions)
        positions.view(-1)[at] = 50
        sa.cache_append(cache, k, k, table, kv_len, rotary=rotary._replace(positions=positions), workspace=ws)
        assert sa.read_status(ws) == sa.E_BAD_INDEX
