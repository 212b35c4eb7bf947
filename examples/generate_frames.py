"""Frames made one after another, as an auto-regressive video generator's attention layer sees them: every step's keys go into a paged
E4M3 cache (normalised, and rotated by the token's time, row and column, with the queries), and its queries attend to all frames so far, the
step's own included; or through a window of the last frames, with the first ones that stay visible, so that a stream of any length takes a
bounded number of pages.  Several streams, of different ages, share the pool and the calls; --fork lets one go on from another's frames.

    python examples/generate_frames.py [--streams 2] [--frames 5] [--grid 30 52] [--heads 12] [--kv-heads 12] [--bf16] [--window 0] [--sink 0] [--fork]

The queries, keys and values of a step are random; the last step is checked against softmax attention in 64 bits over the very numbers that
the cache holds.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2609_23153_b200 as sa


def rotary_tables(d, rows, device):
    """cos, sin [rows, d/2] and the axis of each pair: 22 pairs of 64 turn by the frame, 21 each by the row and the column (other d: alike)."""
    y = x = d // 6
    t = d // 2 - y - x
    freq = torch.cat([10000.0 ** (-torch.arange(n, dtype=torch.float64) / n) for n in (t, y, x)])
    axis = torch.cat([torch.full((n,), a, dtype=torch.int32) for a, n in enumerate((t, y, x))])
    angle = torch.arange(rows, dtype=torch.float64)[:, None] * freq
    return angle.cos().float().to(device), angle.sin().float().to(device), axis.to(device)


class Streams:
    """A pool of pages, the book of who holds which, and how many tokens each stream has."""

    def __init__(self, streams, heads, d, page, tokens, pages, fp8, device):
        """tokens: of the longest stream; pages: of the pool."""
        self.page, self.len, self.device = page, [0] * streams, device
        self.cache = sa.alloc_cache(pages, heads, page, d, fp8=fp8, device=device)
        self.table = torch.full((streams, -(-tokens // page)), -1, dtype=torch.int32, device=device)
        self.refs = torch.zeros(pages, dtype=torch.int32, device=device)

    def lengths(self):
        return torch.tensor(self.len, dtype=torch.int32, device=self.device)

    def grow(self, new):
        """Room for new[b] more tokens of stream b; the step's page table, lengths and row starts on the device."""
        before = self.lengths()
        starts = [0]
        for b, n in enumerate(new):
            self.len[b] += n
            starts.append(starts[-1] + n)
        kv_len = self.lengths()
        _, _, src, dst = sa.pages_reserve(self.table, before, self.refs, kv_len, self.page, page_table_out=self.table, refs_out=self.refs, check_status=True)
        sa.cache_copy_pages(self.cache, src, dst)          # (once for every layer's cache)
        return self.table, kv_len, torch.tensor(starts, dtype=torch.int32, device=self.device)

    def trim(self, frame_tokens, window, sink):
        """What no later frame sees goes back to the pool."""
        sa.pages_trim(self.table, self.lengths(), self.refs, self.page, frame_tokens=frame_tokens, window=window, sink=sink, page_table_out=self.table,
                      refs_out=self.refs)

    def fork(self, parent):
        """Stream b goes on from what stream parent[b] has."""
        self.table, _, self.refs = sa.pages_fork(self.table, self.lengths(), self.refs, torch.tensor(parent, dtype=torch.int32, device=self.device))
        self.len = [self.len[p] for p in parent]


def dense(q, cache, pages, tokens, scale):
    """Softmax attention in 64 bits of the rows q [n, H, d], which see a stream's tokens `tokens`."""
    Hk, page, d = cache.k.shape[1:]
    at, slot = pages[tokens // page].long(), tokens % page

    def rows(x, s):
        y = x.view(torch.uint8)[at, :, slot].view(torch.float8_e4m3fn).double() * s[at].double()[:, :, None] if s is not None else x[at, :, slot].double()
        return y.transpose(0, 1)

    k, v = rows(cache.k, cache.k_scale), rows(cache.v, cache.v_scale)
    a = torch.einsum("nhgd,hjd->hgnj", q.double().view(q.shape[0], Hk, -1, d), k) * scale
    return torch.einsum("hgnj,hjd->nhgd", a.softmax(-1), v).reshape(q.shape)


def run(streams=2, frames=5, grid=(30, 52), heads=12, kv_heads=12, d=128, page=64, fp8=True, window=0, sink=0, fork=False, device="cuda:0",
        check_rows=64, say=print):
    tokens = grid[0] * grid[1]
    gen = torch.Generator(device=device).manual_seed(0)
    longest = (frames + 1) * tokens
    seen = min(longest, sink + (window + 2) * tokens) if window else longest      # what a stream holds at most, with the step's frames
    pool = Streams(streams, kv_heads, d, page, longest, streams * (-(-seen // page) + 3), fp8, device)
    norm = sa.Norm(*(1.0 + 0.2 * torch.randn(d, generator=gen, device=device) for _ in range(2)))
    cos, sin, axis = rotary_tables(d, max(frames + 1, *grid), device)
    cell = torch.arange(tokens, device=device)
    place = torch.stack([torch.zeros_like(cell), cell // grid[1], cell % grid[1]], 1).int()
    workspace = None
    made = [0] * streams
    for step in range(frames):
        # stream 0 makes a frame a step; the others begin with two at once, and pause in the last step but one
        counts = [1 if b == 0 else 2 if step == 0 else 0 if step == frames - 2 else 1 for b in range(streams)]
        table, kv_len, q_start = pool.grow([c * tokens for c in counts])
        positions = torch.cat([place + torch.tensor([[made[b] + f, 0, 0]], dtype=torch.int32, device=device) for b, c in enumerate(counts) for f in range(c)])
        made = [m + c for m, c in zip(made, counts)]
        T = positions.shape[0]
        q, k, v = (torch.randn((T, h, d), generator=gen, device=device).bfloat16() for h in (heads, kv_heads, kv_heads))
        rotary = sa.Rotary(cos, sin, positions=positions, axis=axis, interleaved=True)
        batch = dict(q_start=q_start, max_new=max(counts) * tokens)
        ev = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
        ev[0].record()
        sa.cache_append(pool.cache, k, v, table, kv_len, q=q, q_out=q, norm=norm, rotary=rotary, **batch)
        out = sa.cache_fwd(q, pool.cache, table, kv_len, frame_tokens=tokens, window=window, sink=sink, **batch)
        ev[1].record()
        torch.cuda.synchronize(device)
        say(f"step {step}: {counts} frames, {pool.len} tokens, {int((pool.refs > 0).sum())} pages, {ev[0].elapsed_time(ev[1]):.3f} ms")
        if step < frames - 1:
            pool.trim(tokens, window, sink)
            if fork and streams > 1 and step == frames // 2:
                pool.fork([0, 0] + list(range(2, streams)))        # stream 1 goes another way from stream 0's frames
                made[1] = made[0]
    worst = 0.0
    for b, c in enumerate(counts):
        if c == 0:
            continue
        rows = torch.linspace(0, tokens - 1, min(check_rows, tokens)).long().to(device) + (int(q_start[b + 1]) - tokens)      # of the newest frame
        lo = max(0, pool.len[b] - window * tokens) if window else 0
        at = torch.cat([torch.arange(min(sink, lo), device=device), torch.arange(lo, pool.len[b], device=device)])
        want = dense(q[rows], pool.cache, table[b], at, d ** -0.5)
        worst = max(worst, math.sqrt(float((out[rows].double() - want).square().mean() / want.square().mean())))
    say(f"newest frame against softmax attention in 64 bits over the cache: relative RMS error {worst:.2e}")
    return worst


if __name__ == "__main__":
    p = argparse.ArgumentParser()
    for name, value in (("streams", 2), ("frames", 5), ("heads", 12), ("kv-heads", 12), ("window", 0), ("sink", 0)):
        p.add_argument("--" + name, type=int, default=value)
    p.add_argument("--grid", type=int, nargs=2, default=(30, 52))
    p.add_argument("--bf16", action="store_true")
    p.add_argument("--fork", action="store_true")
    a = p.parse_args()
    sys.exit(run(a.streams, a.frames, tuple(a.grid), a.heads, a.kv_heads, fp8=not a.bf16, window=a.window, sink=a.sink, fork=a.fork) > 1e-2)
