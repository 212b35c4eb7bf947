"""The calls of a generator without end together: pages reserved and copied, keys and queries normalised, rotated and stored, attention through a
window with the first tokens, pages given back; sequences that fork, end, begin again, and a pool that is compacted, step after step against a
plain account of it all."""
import random

import pytest
import torch

import paper_2609_23153_b200 as sa
from examples import generate_frames
from test_gpu_cache import DEV, OUT_RELRMS, check, make_rotary, same_bits
from test_gpu_cache_sink import seen_keys

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Plain:
    """Every sequence's keys and values as they were stored, [H, tokens, d], in 64 bits."""

    def __init__(self, B, H, d):
        self.k, self.v = ([torch.zeros((H, 0, d), dtype=torch.float64, device=DEV) for _ in range(B)] for _ in range(2))

    def fork(self, parent):
        none = torch.zeros_like(self.k[0][:, :0])
        self.k, self.v = ([x[p] if p >= 0 else none for p in parent] for x in (self.k, self.v))

    def attend(self, q, b, length, n, frame, window, sink):
        H, Hk, d = q.shape[1], self.k[b].shape[0], q.shape[2]
        out, lse = torch.zeros(q.shape, dtype=torch.float64, device=DEV), torch.zeros(q.shape[:2], dtype=torch.float64, device=DEV)
        for i in range(n):
            at = torch.tensor(seen_keys(length - n + i, length, frame, window, sink), device=DEV)
            a = torch.einsum("hgd,hjd->hgj", q[i].double().view(Hk, H // Hk, d), self.k[b][:, at]) * d ** -0.5
            lse[i] = torch.logsumexp(a, -1).view(H)
            out[i] = torch.einsum("hgj,hjd->hgd", torch.softmax(a, -1), self.v[b][:, at]).reshape(H, d)
        return out, lse


def stored(cache, row, length):
    """(K, V) of the tokens that a table's row still has, and which these are."""
    P = cache.k.shape[2]
    at = torch.tensor([j for j in range(length) if int(row[j // P]) >= 0], dtype=torch.long, device=DEV)
    pg, slot = row.to(DEV)[at // P].long(), at % P
    got = [x.view(torch.uint8)[pg, :, slot].view(torch.float8_e4m3fn).double() * s[pg].double()[..., None] if s is not None else x[pg, :, slot].double()
           for x, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale))]
    return got[0].transpose(0, 1), got[1].transpose(0, 1), at


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("news,frame,window,sink,page", [((1, 1, 1), 1, 37, 5, 16), ((1, 3, 9), 1, 100, 33, 32), ((20, 40, 20), 20, 3, 20, 16)])
def test_sequences_go_on_fork_and_end(fp8, news, frame, window, sink, page):
    rng = random.Random(window)
    gen = torch.Generator(device=DEV).manual_seed(window)
    B, H, Hk, d, pages, columns, layers = 4, 6, 2, 128, 90, 60, 2
    caches = [sa.alloc_cache(pages, Hk, page, d, fp8=fp8, device=DEV) for _ in range(layers)]
    plain = [Plain(B, Hk, d) for _ in range(layers)]
    table, refs, lens = torch.full((B, columns), -1, dtype=torch.int32, device=DEV), torch.zeros(pages, dtype=torch.int32, device=DEV), [0] * B
    rotary = make_rotary(gen, d, 64, columns * page, 0, 0, True)
    norm = sa.Norm(1 + 0.3 * torch.randn(d, generator=gen, device=DEV), 1 + 0.3 * torch.randn(d, generator=gen, device=DEV))
    steps = 24
    for step in range(steps):
        counts = [rng.choice(news) if n + max(news) <= columns * page and rng.random() < 0.85 else 0 for n in lens]
        if sum(counts) == 0:
            counts[0] = news[0]
        more = [n + c for n, c in zip(lens, counts)]
        before, kv_len, q_start = ints(lens), ints(more), ints([sum(counts[:b]) for b in range(B + 1)])
        _, _, src, dst = sa.pages_reserve(table, before, refs, kv_len, page, page_table_out=table, refs_out=refs, check_status=True)
        lens, T = more, sum(counts)
        for cache, account in zip(caches, plain):
            sa.cache_copy_pages(cache, src, dst, check_status=True)
            q, k, v = (torch.randn((T, h, d), generator=gen, device=DEV).bfloat16() for h in (H, Hk, Hk))
            batch = dict(q_start=q_start, max_new=max(counts), check_status=True)
            rows = sa.cache_append(cache, k, v, table, kv_len, q=q, norm=norm, rotary=rotary, **batch)
            out, lse = sa.cache_fwd(rows, cache, table, kv_len, frame_tokens=frame, window=window, sink=sink, return_lse=True, **batch)
            positions = torch.cat([torch.arange(n - c, n) for n, c in zip(lens, counts)]).int().to(DEV)
            new_k = sa.norm_rotate(k.transpose(0, 1)[None], norm=sa.Norm(norm.k, None), rotary=rotary._replace(positions=positions))[0]
            want, want_lse, t = [], [], 0
            for b, c in enumerate(counts):
                account.k[b] = torch.cat([account.k[b], new_k[:, t:t + c].double()], 1)
                account.v[b] = torch.cat([account.v[b], v[t:t + c].transpose(0, 1).double()], 1)
                if fp8:        # a page's scale grows: what it holds is taken as it is
                    sk, sv, at = stored(cache, table[b].cpu(), lens[b])
                    for mine, its in ((account.k[b], sk), (account.v[b], sv)):
                        # ... and is what was stored to half a step of the code each time its page's scale grew, five times at most here
                        assert ((mine[:, at] - its).abs() <= 2.0 ** -4 * mine[:, at].abs() + 0.05).all()
                        mine[:, at] = its
                else:
                    sk, sv, at = stored(cache, table[b].cpu(), lens[b])
                    assert torch.equal(sk, account.k[b][:, at]) and torch.equal(sv, account.v[b][:, at])
                o, e = account.attend(rows[t:t + c], b, lens[b], c, frame, window, sink)
                want.append(o)
                want_lse.append(e)
                t += c
            check(out, lse, torch.cat(want), torch.cat(want_lse))
        sa.pages_trim(table, kv_len, refs, page, frame_tokens=frame, window=window, sink=sink, page_table_out=table, refs_out=refs, check_status=True)
        if step % 5 == 3:
            parent = [rng.randrange(B) if rng.random() < 0.6 else b for b in range(B)]
            if step % 10 == 8:
                parent[rng.randrange(B)] = -1
            table, kv_len, refs = sa.pages_fork(table, kv_len, refs, ints(parent), check_status=True)
            for account in plain:
                account.fork(parent)
            lens = [lens[p] if p >= 0 else 0 for p in parent]
            assert kv_len.tolist() == lens
        if step % 7 == 5:
            table, refs, src, dst = sa.pages_compact(table, refs, check_status=True)
            for cache in caches:
                sa.cache_copy_pages(cache, src, dst, check_status=True)
            used = int((refs > 0).sum())
            assert (refs[:used] > 0).all() and (refs[used:] == 0).all()
        # the book is the tables', and nobody holds more than what is seen and the pages at its ends
        held = table[table >= 0].long()
        assert torch.equal(refs, torch.bincount(held, minlength=pages).int())
        assert int((table >= 0).sum(1).max()) <= -(-sink // page) + (window + 1) * frame // page + 3
    parent = ints([-1] * B)
    table, _, refs = sa.pages_fork(table, kv_len, refs, parent, check_status=True)
    assert (refs == 0).all() and (table == -1).all()


@pytest.mark.parametrize("kw", [dict(window=3, sink=66, grid=(6, 11), frames=9, heads=4, kv_heads=2, page=16, fork=True), dict(window=2, sink=100, grid=(10, 13), frames=7, fp8=False),
                                dict(window=30, sink=4, grid=(1, 1), frames=120, heads=8, kv_heads=2, page=16, fork=True), dict(grid=(6, 11), frames=6, fork=True)])
def test_example(kw):
    assert generate_frames.run(**dict(dict(streams=3, device=DEV, say=lambda line: None), **kw)) <= OUT_RELRMS


def test_two_calls_at_once():
    """Two batches on two streams, each with its own workspace, have the bits of one after the other."""
    gen = torch.Generator(device=DEV).manual_seed(1)
    made = []
    for i in range(2):
        cache = sa.alloc_cache(40, 2, 32, 128, fp8=bool(i), device=DEV)
        lens = ints([500, 300])
        table = torch.randperm(40, generator=gen, device=DEV).int()[:32].view(2, 16).contiguous()
        k, v = (torch.randn((800, 2, 128), generator=gen, device=DEV).bfloat16() for _ in range(2))
        sa.cache_append(cache, k, v, table, lens, q_start=ints([0, 500, 800]), max_new=500)
        made.append((torch.randn((120, 8, 128), generator=gen, device=DEV).bfloat16(), cache, table, lens))
    args = dict(q_start=ints([0, 100, 120]), max_new=100, window=90, sink=40)
    want = [sa.cache_fwd(*m, **args) for m in made]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in made]
    got = [[sa.cache_fwd(*m, stream=s, **args) for _ in range(5)] for m, s in zip(made, streams)]
    torch.cuda.synchronize()
    assert all(same_bits(x, w) for xs, w in zip(got, want) for x in xs)
