"""Attention over the paged cache where one item's keys lie in many stretches of the line, whose parts the second launch adds up: items of few
and of many rows, beside others of one part."""
import pytest
import torch

import paper_2609_23153_b200 as sa
from test_gpu_cache import DEV, batch_of, check, make_cache, make_table, reference, same_bits

pytestmark = pytest.mark.gpu

CASES = [
    # lens, news, H, Hk, d, page, fp8, frame, window.  Rows of an item: news * H / Hk, up to 128 (17 at least in the longest) or 256 of them
    ([40000], [3], 8, 1, 128, 64, True, 1, 0),
    ([30000], [5], 8, 1, 128, 64, False, 1, 0),
    ([30011], [16], 8, 1, 64, 16, True, 1, 0),
    ([30000], [17], 8, 1, 128, 128, True, 1, 0),
    ([25000], [33], 8, 1, 64, 64, False, 1, 0),
    ([20000], [100], 8, 1, 128, 64, True, 1, 0),
    ([20000], [300], 1, 1, 128, 64, True, 0, 0),
    ([20000, 3, 700, 0], [20, 1, 2, 0], 1, 1, 128, 64, True, 1, 0),         # (20, 1 and 2 rows: sums of a few rows' parts have another order)
    ([9000, 30000, 8], [1, 2, 70], 1, 1, 128, 64, True, 1, 0),              # few rows, many parts, in a call of many rows
    ([9000, 30000, 8], [1, 15, 300], 1, 1, 64, 32, False, 1, 0),
    ([30000, 100], [11, 24], 2, 1, 128, 64, False, 1, 0),
    ([16000, 15000], [40, 17], 8, 2, 128, 64, True, 40, 200),
    ([33000, 5], [5, 5], 8, 1, 128, 64, True, 1, 25000),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) for x in c))
def test_items_of_many_parts(case):
    lens, news, H, Hk, d, page, fp8, frame, window = case
    gen = torch.Generator(device=DEV).manual_seed(sum(lens))
    pages = sum(-(-n // page) for n in lens) + 3
    table = make_table(gen, lens, page, pages)
    cache = make_cache(gen, pages, Hk, page, d, fp8)
    q = torch.randn((sum(news), H, d), generator=gen, device=DEV).bfloat16()
    kv_len, q_start = batch_of(lens, news)
    args = dict(q_start=q_start, max_new=max(news), frame_tokens=frame, window=window, return_lse=True)
    ws = torch.full((1 << 28,), 0xA5, dtype=torch.uint8, device=DEV)
    out, lse = sa.cache_fwd(q, cache, table, kv_len, workspace=ws, **args)
    assert sa.read_status(ws) == (sa.E_BAD_INDEX if any(n > length for length, n in zip(lens, news)) else sa.OK)      # (more new tokens than there are)
    want, want_lse = reference(q, cache, table, lens, news, frame, window)
    check(out, lse, want, want_lse)
    again = sa.cache_fwd(q, cache, table, kv_len, **args)
    assert same_bits(again[0], out) and same_bits(again[1], lse)


def device_us(call, calls=8):
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(calls):
            call()
    times = []
    for _ in range(7):
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        graph.replay()
        b.record()
        torch.cuda.synchronize()
        times.append(a.elapsed_time(b) * 1e3 / calls)
    return sorted(times)[3]


def test_adding_up_many_parts_does_not_set_the_time():
    """131,072 keys of one head, some 148 parts.  Of 32 tokens of 8 heads, 256 rows, they are six times those of 5 tokens, which 1.2 times the time
    pays for; by the CTAs of one border alone it was 1.75 times."""
    gen = torch.Generator(device=DEV).manual_seed(1)
    pages = 2048
    cache = make_cache(gen, pages, 1, 64, 128, True)
    table = torch.randperm(pages, generator=gen, device=DEV).int()[None].contiguous()
    kv_len = torch.tensor([pages * 64], dtype=torch.int32, device=DEV)

    def time(n):
        q = torch.randn((n, 8, 128), generator=gen, device=DEV).bfloat16()
        out = torch.empty_like(q)
        return device_us(lambda: sa.cache_fwd(q, cache, table, kv_len, out=out))

    few, many = time(5), time(32)
    print(f"{few:.1f} us, {many:.1f} us")
    assert many <= 1.5 * few
