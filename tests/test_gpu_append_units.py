"""Appends whose sequences begin anywhere in a page, so that some reach a page more than others, in batches of every kind of split: few sequences of one or two
pages, which share their units out by what they reach; a few of many pages; many of a few tokens."""
import random

import pytest
import torch

import paper_2609_23153_b200 as sa
from test_gpu_cache import DEV, append_reference, batch_of, make_cache, make_rotary, make_table, same_bits

pytestmark = pytest.mark.gpu

BATCHES = [
    # sequences, most new tokens, tokens before: at most, H, Hk, d, page, fp8
    (1, 9, 0, 8, 1, 128, 128, True),
    (1, 128, 200, 2, 2, 64, 128, False),
    (4, 108, 0, 16, 4, 128, 128, True),
    (9, 60, 70, 4, 4, 64, 64, True),
    (20, 17, 40, 3, 1, 128, 16, False),
    (33, 33, 64, 6, 2, 64, 32, True),
    (7, 128, 500, 40, 8, 64, 128, True),
    (3, 300, 90, 12, 12, 64, 64, True),
    (64, 100, 100, 5, 5, 64, 64, False),
    (200, 20, 30, 2, 1, 64, 16, True),
    (150, 3, 30, 8, 8, 64, 16, True),
]


@pytest.mark.parametrize("batch", BATCHES, ids=lambda b: "-".join(str(x) for x in b))
@pytest.mark.parametrize("norm", [False, True])
def test_bits_wherever_sequences_begin(batch, norm):
    B, most, before, H, Hk, d, page, fp8 = batch
    rng = random.Random(B * most)
    gen = torch.Generator(device=DEV).manual_seed(B + most)
    news = [most] + [rng.choice((0, most, rng.randint(1, most))) for _ in range(B - 1)]
    olds = [rng.choice((0, rng.randint(0, before), rng.randint(0, before) // page * page, page - 1)) for _ in range(B)]
    lens = [o + n for o, n in zip(olds, news)]
    pages = sum(-(-n // page) for n in lens) + 2
    cache, table = make_cache(gen, pages, Hk, page, d, fp8), make_table(gen, lens, page, pages)
    kv_len, q_start = batch_of(lens, news)
    T = sum(news)
    q, k, v = ((torch.randn((T, h, d), generator=gen, device=DEV) * torch.exp(torch.randn((T, h, 1), generator=gen, device=DEV))).bfloat16() for h in (H, Hk, Hk))
    rotary = make_rotary(gen, d, 64, max(lens) + 1, T, 0, False)
    weights = sa.Norm(*(1 + 0.5 * torch.randn(d, generator=gen, device=DEV) for _ in range(2))) if norm else None
    if norm:
        # each row has the bits of the call over whole sequences; over E4M3 pages the largest values decide, so the row is compared, not its codes
        want_q = sa.norm_rotate(q.transpose(0, 1)[None].contiguous(), norm=weights, rotary=rotary._replace(positions=torch.cat(
            [torch.arange(o, o + n) for o, n in zip(olds, news)]).int().to(DEV)))[0].transpose(0, 1)
        want = None
    else:
        want, want_q = append_reference(cache, k, v, table, lens, news, rotary, q)
    others = [None if x is None else x.clone() for x in cache]
    got_q = sa.cache_append(cache, k, v, table, kv_len, q_start=q_start, max_new=max(news), q=q, norm=weights, rotary=rotary, check_status=True)
    assert same_bits(got_q, want_q)
    if not norm:
        for got, ref in zip(cache, want):
            assert got is None or same_bits(got, ref)
        return
    # one sequence at a time: the same bits, page by page
    for b in range(B):
        if news[b]:
            at = slice(int(q_start[b]), int(q_start[b + 1]))
            sa.cache_append(sa.KVCache(*others), k[at], v[at], table[b:b + 1].contiguous(), kv_len[b:b + 1].contiguous(), norm=weights, rotary=rotary)
    for got, ref in zip(cache, others):
        assert got is None or same_bits(got, ref)
