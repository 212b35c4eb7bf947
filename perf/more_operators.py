"""The work of a generator that goes on for long over a paged key/value cache, as cases that can be timed and compared.

  whole    norm of each head's query and key and their rotation, in one pass over a whole sequence (in front of the block-sparse attention)
  append   the same for new tokens on their way into the cache: bf16, or E4M3 with one scale per page and head
  attend   softmax attention of the new tokens over the cache, through a sliding window of frames (or tokens) and the sequence's first
           tokens, which stay visible
  fork     sequences of the next step go on from sequences of this one: page tables gathered, the pages' users counted
  reserve  pages for new tokens; a partly filled page that several sequences hold is copied for all but one
  trim     pages that no later token reads are given back
  compact  the pages in use move to the front of the pool

Batches are ragged: sequence b owns the tokens q_start[b] .. q_start[b+1] - 1 of a call and kv_len[b] tokens of the cache, the
new ones included.  Lengths follow from the case alone; values, page order and rotary phases from the seed.

`run` computes the operators with this package's calls where `own` is true, and else with elementary torch operations.
"""
import math

import torch

own = False

E4M3_MAX = 448.0
FRAME_480P = (30, 52)        # latent grid of a 480 x 832 frame: 1560 tokens
LARGEST_FLOPS = 1.0e12
LARGEST_BYTES = 3.2e9


def listed():
    def norm(name, op, **more):
        return dict(name=name, op=op, batch=1, heads=12, kv_heads=12, dim=128, rot=128, axes=1, interleaved=False, weight="float32", per_head=False, new=1, old=0,
                    ragged=False, page=64, fp8=True, grid_h=30, grid_w=52, heads_inner=False) | more

    def attend(name, batch, length, new, heads, kv_heads, page, fp8, window, sink, **more):
        return dict(name=name, op="attend", batch=batch, length=length, new=new, ragged=False, hole=False, heads=heads, kv_heads=kv_heads, dim=128, page=page,
                    fp8=fp8, frame=1, window=window, sink=sink) | more

    def book(name, op, batch, length, page, share, **more):
        return dict(name=name, op=op, batch=batch, length=length, page=page, share=share, new=1, spare=64, window=0, sink=0, frame=1, kv_heads=0, dim=128,
                    fp8=True) | more

    return [
        # the 14B model's layer at 720P: 40 heads over 21 x 45 x 80 latent tokens, rotated by (t, y, x)
        norm("whole_720p", "whole", heads=40, kv_heads=40, new=75600, axes=3, interleaved=True, grid_h=45, grid_w=80),
        # a short odd sequence of two samples, heads of 64 channels stored token by token, fewer key heads, weights of each head
        norm("whole_short", "whole", batch=2, heads=6, kv_heads=2, dim=64, rot=32, new=1201, weight="bfloat16", per_head=True, heads_inner=True),
        # a serving step: a token for each of many sequences, the last pages partly filled
        norm("append_step", "append", batch=128, old=2047, heads=40, kv_heads=8, ragged=True),
        # three latent frames at 480P enter the cache of the 1.3B model's layer
        norm("append_frames", "append", old=9360, new=4680, page=128, axes=3, interleaved=True, weight="bfloat16"),
        # one conversation of thirty thousand tokens, of which a thousand and the first four are seen: latency
        attend("sink_one", 1, 30001, 1, 32, 8, 64, True, 1000, 4),
        # a serving step over sequences of very different lengths, most of them far longer than what is seen
        attend("sink_step", 32, 16383, 1, 40, 8, 64, True, 4000, 64, ragged=True),
        # three latent frames at 480P see five frames up to their own, and the first
        attend("sink_frames", 1, 32760, 4680, 12, 12, 128, True, 5, 1560, frame=1560),
        # a piece of each of four prompts over bf16 pages
        attend("sink_prompts", 4, 8000, 2048, 32, 8, 64, False, 1500, 100, ragged=True),
        # a step of a search with four continuations of each of 64 prompts: all rows change places
        book("fork_beams", "fork", 256, 32000, 64, 4, spare=4000),
        # a token for each of 128 sequences, fours of which have just been forked: pages, and copies of what they share
        book("reserve_step", "reserve", 128, 8191, 16, 4, kv_heads=8),
        # frames leave the window of 32 video streams
        book("trim_frames", "trim", 32, 60000, 128, 1, frame=1560, window=7, sink=1560),
        # half of the pool of a 1.3B model's layer has been given back: the rest moves together
        book("compact_pool", "compact", 8, 16380, 128, 1, spare=1000, kv_heads=12),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(("whole", "append", "attend", "attend", "fork", "reserve", "trim", "compact"))
        kv_heads = rng.choice((1, 2, 4, 8, 12))
        c = dict(op=op, kv_heads=kv_heads, heads=kv_heads * rng.choice((1, 1, 2, 3, 4, 5, 7, 8, 12, 16)), dim=rng.choice((64, 128, 128)),
                 page=rng.choice((16, 32, 64, 128)), fp8=rng.random() < 0.7, ragged=rng.random() < 0.6)
        if c["heads"] > 64:
            continue
        if op in ("whole", "append"):
            frames = rng.random() < 0.4
            c.update(rot=rng.choice((c["dim"], c["dim"] // 2)), axes=3 if frames else 1, interleaved=frames or rng.random() < 0.3,
                     weight=rng.choice(("float32", "bfloat16")), per_head=rng.random() < 0.3, grid_h=rng.randint(4, 45), grid_w=rng.randint(4, 80),
                     heads_inner=rng.random() < 0.5)
            if op == "whole":
                c.update(batch=rng.randint(1, 4), new=_log_int(rng, 1, 80000), old=0, ragged=False)
            else:
                c.update(batch=_log_int(rng, 1, 128), old=rng.choice((0, _log_int(rng, 1, 4000))), new=1 if rng.random() < 0.4 else _log_int(rng, 2, 6000))
            if c["batch"] * c["new"] * c["heads"] * c["dim"] > 4.0e8:
                continue
        elif op == "attend":
            kind = rng.random()
            new = 1 if kind < 0.5 else rng.randint(2, 16) if kind < 0.65 else _log_int(rng, 17, 4700)
            frame = 1 if kind < 0.65 or rng.random() < 0.5 else _log_int(rng, 16, 1560)
            length = new + _log_int(rng, 1, 131072)
            window = max(1, _log_int(rng, 1, length) // frame)
            batch = _log_int(rng, 1, 128)
            c.update(batch=batch, length=length, new=new, hole=batch > 1 and rng.random() < 0.2, frame=frame, window=window,
                     sink=rng.choice((1, 4, _log_int(rng, 1, 4096), frame)))
            if batch * c["heads"] * new * length > 2.0e9 or batch * length * kv_heads * c["dim"] > 4.0e8:
                continue
        else:
            share = 1 if op in ("trim", "compact") else rng.choice((1, 2, 4, 5))
            frame = rng.choice((1, _log_int(rng, 16, 1560))) if op == "trim" else 1
            c.update(batch=share * _log_int(rng, 1, 256 // share), length=_log_int(rng, 1, 65536), share=share, spare=_log_int(rng, 1, 4000), frame=frame,
                     new=1 if rng.random() < 0.5 else _log_int(rng, 2, 4000), sink=rng.choice((0, 4, frame)) if op == "trim" else 0,
                     window=max(1, _log_int(rng, 1, 20000) // frame) if op == "trim" else 0)
            if op in ("fork", "trim"):
                c.update(kv_heads=0)
            if op == "compact":
                c.update(spare=max(c["spare"], 8))
            pages, moved = _pages(c), c["kv_heads"] * c["page"] * c["dim"] * (1 if c["fp8"] else 2)
            if pages * moved > 4.0e8 or pages > 400000:
                continue
        w = work(c)
        if w["flops"] <= LARGEST_FLOPS and w["bytes"] <= LARGEST_BYTES:
            return c


# ------------------------------------------------------------------------------------------------------------- lengths and work

def _lengths(case):
    """(tokens in the cache, new tokens among them) of every sequence."""
    got = []
    for b in range(case["batch"]):
        f = 1.0 if b == 0 or not case["ragged"] else (b * 0.6180339887498949) % 1.0
        new = max(1, math.ceil(case["new"] * f))
        if case["op"] == "append":
            got.append((new + math.floor(case["old"] * f), new))
        else:
            hole = case["hole"] and b == case["batch"] // 2
            got.append((0 if hole else max(new, math.ceil(case["length"] * f)), new))
    return got


def _seen(case, length, new):
    """[first, last) of the window of each new token of a sequence, and the end of the first tokens that it sees besides."""
    g, w, rows = case["frame"], case["window"], []
    for pos in range(length - new, length):
        if pos < 0:
            rows.append((0, 0, 0))
        else:
            hi = min(length, (pos // g + 1) * g)
            lo = min(hi, max(0, (pos // g - w + 1) * g))
            rows.append((lo, hi, min(case["sink"], lo)))
    return rows


def _held(case):
    """Tokens that every sequence of a book has, before what is new.  Groups of `share` have the same."""
    got = []
    for b in range(case["batch"]):
        f = 1.0 if b < case["share"] else (b // case["share"] * 0.6180339887498949) % 1.0
        got.append(max(1, math.ceil(case["length"] * f)))
    return got


def _more(case):
    """... and with it."""
    return [n + max(1, math.ceil(case["new"] * (1.0 if b % 3 == 0 else 0.4))) for b, n in enumerate(_held(case))]


def _pages(case):
    """Pages of a book's pool: those in use, what is reserved, and some to spare."""
    P, share = case["page"], case["share"]
    held, more = _held(case), _more(case)
    used = sum(-(-n // P) for n in held[::share])
    return used + sum(-(-m // P) - -(-n // P) + 1 for n, m in zip(held, more)) + case["spare"]


def _columns(case):
    return max(-(-m // case["page"]) for m in _more(case)) + 1


def work(case):
    op, d = case["op"], case["dim"]
    size = 1 if case["fp8"] else 2
    if op in ("whole", "append"):
        H, Hk, weights = case["heads"], case["kv_heads"], (case["heads"] + case["kv_heads"] if case["per_head"] else 2) * d * (4 if case["weight"] == "float32" else 2)
        flops = lambda rows: rows * (5 * d + 3 * case["rot"])
        if op == "whole":
            T = case["batch"] * case["new"]
            table = min(case["new"], 64 + case["new"] if case["axes"] == 1 else 512) * case["rot"] * 4 + (12 * case["new"] if case["axes"] == 3 else 0)
            return {"bytes": 4 * T * d * (H + Hk) + table + weights, "flops": flops(T * (H + Hk))}
        lens = _lengths(case)
        T = sum(n for _, n in lens)
        positions = max(length for length, _ in lens) if case["axes"] == 1 else T
        touched = sum((length - 1) // case["page"] - (length - n) // case["page"] + 1 for length, n in lens)
        moved = T * d * (2 * 2 * H + 2 * 2 * Hk + 2 * size * Hk) + weights
        moved += min(T, positions) * case["rot"] * 4 + 4 * T * case["axes"] + 4 * touched * (1 + (2 * Hk if case["fp8"] else 0))
        return {"bytes": moved, "flops": flops(T * (H + Hk))}
    if op == "attend":
        H, Hk, P = case["heads"], case["kv_heads"], case["page"]
        lens = _lengths(case)
        T, pairs, keys, pages = sum(n for _, n in lens), 0, 0, 0
        for length, n in lens:
            rows = _seen(case, length, n)
            pairs += sum(hi - lo + s for lo, hi, s in rows)
            lo, hi, s = min((r[0] for r in rows if r[1] > 0), default=0), max((r[1] for r in rows), default=0), max((r[2] for r in rows), default=0)
            keys += hi - lo + min(s, lo)
            pages += -(-hi // P) - lo // P + -(-min(s, lo) // P)
        moved = keys * Hk * 2 * d * size + T * H * (2 * 2 * d + 4) + 4 * pages + (8 * pages * Hk if case["fp8"] else 0)
        return {"bytes": moved, "flops": 4 * d * H * pairs}
    # books: the tables' and counts' words, and the pages that move
    B, P, pages, share = case["batch"], case["page"], _pages(case), case["share"]
    held, more = _held(case), _more(case)
    entries = sum(-(-n // P) for n in held)
    page_bytes = 2 * case["kv_heads"] * (P * d * size + (4 if case["fp8"] else 0))
    moved = 8 * entries + 8 * pages + 12 * B
    if op == "reserve":
        copies = sum(n % P != 0 and b % share != 0 for b, n in enumerate(held))
        moved += 2 * copies * page_bytes + 8 * B
    if op == "compact":
        moved += 2 * int(entries * (1.0 - entries / pages)) * page_bytes
    return {"bytes": moved, "flops": B * _columns(case)}


# ------------------------------------------------------------------------------------------------------------------ inputs

def _power_scale(amax):
    """The smallest power of two s with amax <= 448 s, as the cache's scales are."""
    mantissa, exponent = torch.frexp(amax.clamp(min=1e-12))        # mantissa in [0.5, 1); 448 = 0.875 * 2^9
    return torch.ldexp(torch.ones_like(amax), exponent - 9 + (mantissa > 0.875).int())


def _filled(shape, fp8, gen):
    """(pages of keys or values, their scales): normal values whose channels and heads differ in size."""
    pages, heads, page, d = shape
    x = torch.randn(shape, generator=gen, device="cuda")
    x *= torch.exp(0.5 * torch.randn((1, heads, 1, d), generator=gen, device="cuda"))
    if not fp8:
        return x.bfloat16(), None
    scale = _power_scale(x.abs().amax(dim=(2, 3)))
    x /= scale[:, :, None, None]
    return x.to(torch.float8_e4m3fn), scale


def _pools(case, pages, gen):
    shape = (pages, case["kv_heads"], case["page"], case["dim"])
    s = {}
    s["k_cache"], s["k_scale"] = _filled(shape, case["fp8"], gen)
    s["v_cache"], s["v_scale"] = _filled(shape, case["fp8"], gen)
    return s


def _rows(shape, gen):
    """bf16 rows [..., heads, d] as a projection leaves them: channels differ in size, and so do tokens."""
    x = torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16)
    x *= torch.exp(0.7 * torch.randn(shape[-2:], generator=gen, device="cuda")).bfloat16()
    x *= torch.exp(0.5 * torch.randn(shape[:-2] + (1, 1), generator=gen, device="cuda")).bfloat16()
    return x


def _norm_inputs(case, positions, longest, gen):
    """Weights, and tables of the rotation; `positions`: of the call's tokens in their sequences."""
    dev, d = "cuda", case["dim"]
    dtype = getattr(torch, case["weight"])
    s = {}
    for name, heads in (("q_weight", case["heads"]), ("k_weight", case["kv_heads"])):
        s[name] = (1.0 + 0.3 * torch.randn((heads, d) if case["per_head"] else (d,), generator=gen, device=dev)).to(dtype)
    pairs = case["rot"] // 2
    phase = torch.rand((), generator=gen, device=dev).double()
    if case["axes"] == 3:        # thirds of the pairs turn with t, y and x of the token on the latent grid
        third = -(-pairs // 3)
        axis = torch.tensor([min(m // third, 2) for m in range(pairs)], dtype=torch.int32)
        freq = torch.tensor([10000.0 ** (-(m % third) / third) for m in range(pairs)], dtype=torch.float64)
        hg, wg = case["grid_h"], case["grid_w"]
        s["positions"] = torch.stack([positions // (hg * wg), positions // wg % hg, positions % wg], dim=1).int().to(dev)
        s["axis"] = axis.to(dev)
        rows = max(longest // (hg * wg) + 1, hg, wg)
    else:
        freq = torch.tensor([10000.0 ** (-m / pairs) for m in range(pairs)], dtype=torch.float64)
        s["positions"] = s["axis"] = None
        rows = longest
    angle = torch.arange(rows, device=dev)[:, None].double() * freq.to(dev)[None] + phase
    s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
    return s


def _prepare_whole(case, gen):
    B, N, d = case["batch"], case["new"], case["dim"]
    s = _norm_inputs(case, torch.arange(N), N, gen)
    for name, heads in (("q", case["heads"]), ("k", case["kv_heads"])):
        x = _rows((B, N, heads, d), gen).transpose(1, 2)
        s[name] = x if case["heads_inner"] else x.contiguous()
    return s


def _batch_of(case, gen):
    """Lengths, starts and a page table whose pages lie in the pool in no order."""
    lens, P, dev = _lengths(case), case["page"], "cuda"
    starts = [0]
    for _, n in lens:
        starts.append(starts[-1] + n)
    need = [-(-length // P) for length, _ in lens]
    pages = sum(need) + 3
    order = torch.randperm(pages, generator=gen, device=dev).int().cpu()
    table = torch.zeros((case["batch"], max(need) + 1), dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return pages, {"page_table": table.to(dev), "kv_len": torch.tensor([length for length, _ in lens], dtype=torch.int32, device=dev),
                   "q_start": torch.tensor(starts, dtype=torch.int32, device=dev), "max_new": max(n for _, n in lens)}


def _prepare_rows(case, gen):
    lens = _lengths(case)
    pages, s = _batch_of(case, gen)
    T = sum(n for _, n in lens)
    s.update(_pools(case, pages, gen))
    if case["op"] == "attend":
        s["q"] = (1.5 * torch.randn((T, case["heads"], case["dim"]), generator=gen, device="cuda")).bfloat16()
        return s
    s["q"], s["k"] = _rows((T, case["heads"], case["dim"]), gen), _rows((T, case["kv_heads"], case["dim"]), gen)
    s["v"] = (1.5 * torch.randn((T, case["kv_heads"], case["dim"]), generator=gen, device="cuda")).bfloat16()
    s.update(_norm_inputs(case, torch.cat([torch.arange(length - new, length) for length, new in lens]), max(length for length, _ in lens), gen))
    return s


def _prepare_book(case, gen):
    """Sequences in groups of `share` that hold the same pages, in a pool in no order."""
    dev, P, share, B = "cuda", case["page"], case["share"], case["batch"]
    held, pages = _held(case), _pages(case)
    order = torch.randperm(pages, generator=gen, device=dev).int().cpu()
    table = torch.full((B, _columns(case)), -1, dtype=torch.int32)
    refs = torch.zeros(pages, dtype=torch.int32)
    at = 0
    for b, n in enumerate(held):
        need = -(-n // P)
        if b % share == 0:
            mine = order[at:at + need]
            at += need
        table[b, :need] = mine
        refs[mine.long()] += 1
    s = {"page_table": table.to(dev), "refs": refs.to(dev), "kv_len": torch.tensor(held, dtype=torch.int32, device=dev)}
    if case["op"] == "fork":        # beams take each other's places within their group; some sequences end, some begin twice
        group = torch.arange(B, device=dev) // share * share
        s["parent"] = (group + torch.randint(0, share, (B,), generator=gen, device=dev)).int()
        s["parent"][torch.rand(B, generator=gen, device=dev) < 0.05] = -1
    if case["op"] == "reserve":
        s["kv_new"] = torch.tensor(_more(case), dtype=torch.int32, device=dev)
    if case["op"] in ("reserve", "compact"):
        s.update(_pools(case, pages, gen))
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    make = {"whole": _prepare_whole, "append": _prepare_rows, "attend": _prepare_rows}.get(case["op"], _prepare_book)
    return dict(make(case, gen), case=dict(case))


# --------------------------------------------------------------------------------------------------------------- plain forms

def _owners(s):
    """(sequence, position in it) of every token of the call."""
    token = torch.arange(s["q"].shape[0], device="cuda")
    seq = torch.searchsorted(s["q_start"][1:].long(), token, right=True)
    return seq, s["kv_len"].long()[seq] - (s["q_start"].long()[seq + 1] - token)


def _normed(x, weight, eps=1e-6):
    x = x.float()
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + eps) * weight.float()


def _rotate(x, cos, sin, interleaved):
    """x [..., d] with the first 2 * cos.shape[-1] channels turned by the angles of cos, sin [..., pairs]."""
    rot = 2 * cos.shape[-1]
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], dim=-1)
    return torch.cat([turned, x[..., rot:]], dim=-1)


def _phases(s, pos):
    if s["positions"] is None:
        return s["cos"][pos], s["sin"][pos]
    at = s["positions"].long()[:, s["axis"].long()]                # [T, pairs]
    return s["cos"].gather(0, at), s["sin"].gather(0, at)


def _plain_whole(s):
    c = s["case"]
    cos, sin = _phases(s, torch.arange(c["new"], device="cuda"))

    def turned(x, weight):
        return _rotate(_normed(x, weight[:, None] if c["per_head"] else weight), cos, sin, c["interleaved"]).bfloat16()

    return {"q": turned(s["q"], s["q_weight"]), "k": turned(s["k"], s["k_weight"])}


def _e4m3(x):
    return x.clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).view(torch.uint8)


def _store_fp8(s, x, cache, scale, page, slot):
    """x [T, heads, d] into an E4M3 cache: a page's scale only grows while it fills, and what it holds is encoded again then."""
    P = s["case"]["page"]
    bytes_ = cache.view(torch.uint8)
    fresh = _power_scale(torch.zeros_like(scale).index_reduce_(0, page, x.abs().amax(-1), "amax"))
    before = s["kv_len"].long() - (s["q_start"][1:] - s["q_start"][:-1]).long()          # tokens that were there
    first = s["page_table"].long().gather(1, (before // P)[:, None])[:, 0]                # the only page that may be partly filled
    held = (before % P)[:, None]
    old = scale[first]
    grown = torch.where(held > 0, torch.maximum(old, fresh[first]), fresh[first])
    touched = torch.zeros(scale.shape[0], dtype=torch.bool, device="cuda").index_fill_(0, page, True)
    scale.copy_(torch.where(touched[:, None], fresh, scale))
    scale[first] = grown
    again = _e4m3(cache[first].float() * (old * (1.0 / grown))[:, :, None, None])
    keep = (torch.arange(P, device="cuda")[None] >= held)[:, None] | (old >= grown)[:, :, None]
    bytes_[first] = torch.where(keep[..., None], bytes_[first], again)
    bytes_[page, :, slot] = _e4m3(x * (1.0 / scale[page])[:, :, None])


def _plain_append(s):
    c = s["case"]
    seq, pos = _owners(s)
    cos, sin = (x[:, None] for x in _phases(s, pos))
    q, k, v = _rotate(_normed(s["q"], s["q_weight"]), cos, sin, c["interleaved"]), _rotate(_normed(s["k"], s["k_weight"]), cos, sin, c["interleaved"]), s["v"].float()
    page, slot = s["page_table"].long()[seq, pos // c["page"]], pos % c["page"]
    if c["fp8"]:
        _store_fp8(s, k, s["k_cache"], s["k_scale"], page, slot)
        _store_fp8(s, v, s["v_cache"], s["v_scale"], page, slot)
    else:
        s["k_cache"][page, :, slot] = k.bfloat16()
        s["v_cache"][page, :, slot] = v.bfloat16()
    return {"q": q.bfloat16()} | {n: s[n] for n in ("k_cache", "v_cache", "k_scale", "v_scale")}


def _plain_attend(s):
    c = s["case"]
    B, n, H, Hk, d, g = c["batch"], s["max_new"], c["heads"], c["kv_heads"], c["dim"], c["frame"]
    G = H // Hk
    columns = s["page_table"].shape[1] - 1
    table = s["page_table"].long()[:, :columns]
    L = columns * c["page"]

    def dense(cache, scale):
        x = cache.view(torch.uint8)[table].view(torch.float8_e4m3fn).float() if c["fp8"] else cache[table].float()
        if scale is not None:
            x *= scale[table][..., None, None]
        return x.permute(0, 2, 1, 3, 4).reshape(B, Hk, L, d)

    start, length = s["q_start"].long()[:-1], s["kv_len"].long()
    count = s["q_start"].long()[1:] - start
    at = (start[:, None] + torch.arange(n, device="cuda")[None]).clamp(max=s["q"].shape[0] - 1)       # [B, n]
    q = s["q"][at].float().reshape(B, n, Hk, G, d).permute(0, 2, 3, 1, 4).reshape(B, Hk, G * n, d)
    scores = torch.matmul(q, dense(s["k_cache"], s["k_scale"]).transpose(2, 3)).view(B, Hk, G, n, L) / math.sqrt(d)
    key = torch.arange(L, device="cuda")[None, None]
    pos = (length - count)[:, None, None] + torch.arange(n, device="cuda")[None, :, None]
    frame = torch.div(pos, g, rounding_mode="floor")
    seen = (key < length[:, None, None]) & (key < (frame + 1) * g) & (pos >= 0) & ((key >= (frame - c["window"] + 1) * g) | (key < c["sink"]))
    scores.masked_fill_(~seen[:, None, None].expand_as(scores), -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(torch.isfinite(top), top, 0.0)
    scores.sub_(top).exp_()
    total = scores.sum(-1, keepdim=True)
    out = torch.matmul(scores.view(B, Hk, G * n, L), dense(s["v_cache"], s["v_scale"])).view(B, Hk, G, n, d)
    out = torch.where(total > 0, out / total, 0.0)
    lse = (top + total.log())[..., 0]
    seq = torch.searchsorted(s["q_start"][1:].long(), torch.arange(s["q"].shape[0], device="cuda"), right=True)
    row = torch.arange(s["q"].shape[0], device="cuda") - start[seq]
    out = out.permute(0, 3, 1, 2, 4).reshape(B, n, H, d)[seq, row]
    return {"out": out.bfloat16(), "lse": lse.permute(0, 3, 1, 2).reshape(B, n, H)[seq, row]}


def _plain_fork(s):
    table, refs, parent = s["page_table"], s["refs"], s["parent"].long()
    there = parent >= 0
    from_ = parent.clamp(min=0)
    uses = torch.zeros(table.shape[0], dtype=torch.int32, device="cuda").index_add_(0, from_, there.int()) - 1
    change = torch.where(table >= 0, uses[:, None], 0).flatten()
    return {"page_table": torch.where(there[:, None], table[from_], -1), "kv_len": torch.where(there, s["kv_len"][from_], 0),
            "refs": refs.index_add(0, table.clamp(min=0).flatten(), change)}


def _copy_pages(s, src, dst):
    src, dst = src[src >= 0].long(), dst[dst >= 0].long()
    for name in ("k_cache", "v_cache"):
        x = s[name].view(torch.uint8) if s["case"]["fp8"] else s[name]
        x[dst] = x[src]
    if s["case"]["fp8"]:
        s["k_scale"][dst] = s["k_scale"][src]
        s["v_scale"][dst] = s["v_scale"][src]
    return {n: s[n] for n in ("k_cache", "v_cache", "k_scale", "v_scale")}


def _plain_reserve(s):
    table, refs, P = s["page_table"], s["refs"], s["case"]["page"]
    B, columns = table.shape
    pages = refs.shape[0]
    old, new = s["kv_len"].long(), s["kv_new"].long()
    tail = (old // P).clamp(max=columns - 1)
    page = table.gather(1, tail[:, None])[:, 0].long()
    shared = (old % P != 0) & (new > old) & (page >= 0) & (refs[page.clamp(min=0)] > 1)
    # whoever comes first keeps a page that only sequences of this call hold
    at = torch.where(shared, page, pages)
    row = torch.arange(B, device="cuda")
    writers = torch.zeros(pages + 1, dtype=torch.long, device="cuda").index_add_(0, at, torch.ones_like(at))
    first = torch.full((pages + 1,), B, dtype=torch.long, device="cuda").scatter_reduce_(0, at, row, "amin")
    copies = shared & ~((writers[at] == refs[page.clamp(min=0)]) & (first[at] == row))
    column = torch.arange(columns, device="cuda")[None]
    asked = (column >= ((old + P - 1) // P)[:, None]) & (column < ((new + P - 1) // P)[:, None]) & (table < 0)
    asked |= (column == tail[:, None]) & copies[:, None]
    rank = (asked.flatten().cumsum(0) - 1).view(B, columns)
    free = refs == 0
    number = torch.where(free, free.cumsum(0) - 1, pages)
    free_pages = torch.zeros(pages + 1, dtype=torch.int32, device="cuda").scatter_(0, number, torch.arange(pages, device="cuda", dtype=torch.int32))
    enough = asked.sum() <= free.sum()
    asked, copies = asked & enough, copies & enough
    given = free_pages[rank.clamp(0, pages)]
    one = asked.flatten().int()
    refs = refs.index_add(0, torch.where(asked, given, 0).flatten(), one).index_add(0, page.clamp(min=0), -copies.int())
    dst = given.gather(1, tail[:, None])[:, 0]
    src, dst = torch.where(copies, page, -1).int(), torch.where(copies, dst, -1)
    return {"page_table": torch.where(asked, given, table), "refs": refs, "src": src, "dst": dst} | _copy_pages(s, src, dst)


def _plain_trim(s):
    c, table, P = s["case"], s["page_table"], s["case"]["page"]
    length = s["kv_len"].long()[:, None]
    lo = (length // c["frame"] - c["window"] + 1) * c["frame"] if c["window"] else torch.zeros_like(length)
    column = torch.arange(table.shape[1], device="cuda")[None]
    dead = ((column * P >= c["sink"]) & ((column + 1) * P <= lo)) | (column * P >= length)
    gone = dead & (table >= 0)
    return {"page_table": torch.where(dead, -1, table), "refs": s["refs"].index_add(0, table.clamp(min=0).flatten(), -gone.flatten().int())}


def _plain_compact(s):
    table, refs = s["page_table"], s["refs"]
    pages = refs.shape[0]
    page = torch.arange(pages, device="cuda")
    used = refs > 0
    front = page < used.sum()
    moves, holes = used & ~front, ~used & front

    def in_order(mask):
        place = torch.where(mask, mask.cumsum(0) - 1, pages)
        return torch.full((pages + 1,), -1, dtype=torch.int32, device="cuda").scatter_(0, place, page.int())[:pages // 2]

    def only(mask, found):        # (what is not in the mask went to the last place)
        return torch.where(torch.arange(found.shape[0], device="cuda") < mask.sum(), found, -1)

    src, dst = only(moves, in_order(moves)), only(holes, in_order(holes))
    to = torch.where(used, page.int(), -1)
    to[src[src >= 0].long()] = dst[dst >= 0]
    after = torch.zeros_like(refs)
    after[to[used].long()] = refs[used]
    return {"page_table": torch.where(table >= 0, to[table.clamp(min=0).long()], -1), "refs": after, "src": src, "dst": dst} | _copy_pages(s, src, dst)


# ------------------------------------------------------------------------------------------------------------------- passes

def _own(s):
    import paper_2609_23153_b200 as sa
    c = s["case"]
    op, P = c["op"], c["page"]
    cache = sa.KVCache(s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"]) if "k_cache" in s else None
    pools = {n: s[n] for n in ("k_cache", "v_cache", "k_scale", "v_scale")} if cache else {}
    if op in ("whole", "append"):
        rotary = sa.Rotary(s["cos"], s["sin"], positions=s["positions"], axis=s["axis"], interleaved=c["interleaved"])
        norm = sa.Norm(s["q_weight"], s["k_weight"])
        if op == "whole":
            q, k = sa.norm_rotate(s["q"], s["k"], norm=norm, rotary=rotary)
            return {"q": q, "k": k}
        q = sa.cache_append(cache, s["k"], s["v"], s["page_table"], s["kv_len"], q=s["q"], norm=norm, rotary=rotary, q_start=s["q_start"], max_new=s["max_new"])
        return {"q": q} | pools
    if op == "attend":
        out, lse = sa.cache_fwd(s["q"], cache, s["page_table"], s["kv_len"], frame_tokens=c["frame"], window=c["window"], sink=c["sink"], return_lse=True,
                                q_start=s["q_start"], max_new=s["max_new"])
        return {"out": out, "lse": lse}
    if op == "fork":
        table, kv_len, refs = sa.pages_fork(s["page_table"], s["kv_len"], s["refs"], s["parent"])
        return {"page_table": table, "kv_len": kv_len, "refs": refs}
    if op == "trim":
        table, refs = sa.pages_trim(s["page_table"], s["kv_len"], s["refs"], P, frame_tokens=c["frame"], window=c["window"], sink=c["sink"])
        return {"page_table": table, "refs": refs}
    if op == "reserve":
        table, refs, src, dst = sa.pages_reserve(s["page_table"], s["kv_len"], s["refs"], s["kv_new"], P)
    else:
        table, refs, src, dst = sa.pages_compact(s["page_table"], s["refs"])
    sa.cache_copy_pages(cache, src, dst)
    return {"page_table": table, "refs": refs, "src": src, "dst": dst} | pools


def run(s):
    if own:
        return _own(s)
    plain = {"whole": _plain_whole, "append": _plain_append, "attend": _plain_attend, "fork": _plain_fork, "reserve": _plain_reserve, "trim": _plain_trim,
             "compact": _plain_compact}
    return plain[s["case"]["op"]](s)


# ------------------------------------------------------------------------------------------------------------ in 64 bits

def _unit64(x, weight):
    x = x.double()
    return x / torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + 1e-6) * weight.double()


def _turned64(x, s, pos):
    """Rows x [..., T, d] of tokens at positions pos [T], in 64 bits."""
    c = s["case"]
    pairs = c["rot"] // 2
    m = torch.arange(pairs, device="cuda")
    p = pos[:, None].expand(-1, pairs) if s["positions"] is None else s["positions"].long()[:, s["axis"].long()]
    w = torch.complex(s["cos"][p, m].double(), s["sin"][p, m].double())
    first, second = (2 * m, 2 * m + 1) if c["interleaved"] else (m, m + pairs)
    z = torch.complex(x[..., first], x[..., second]) * w
    x[..., first], x[..., second] = z.real, z.imag
    return x


def _exact_whole(s):
    got = {}
    pos = torch.arange(s["case"]["new"], device="cuda")
    for name in ("q", "k"):
        x, weight = s[name], s[name + "_weight"]
        y = torch.empty(x.shape, dtype=torch.float64, device="cuda")
        for b in range(x.shape[0]):
            for h in range(x.shape[1]):
                y[b, h] = _turned64(_unit64(x[b, h], weight[h] if weight.dim() == 2 else weight), s, pos)
        got[name] = y
    return got


def _exact_append(s):
    c = s["case"]
    P = c["page"]
    starts, lens, table = s["q_start"].tolist(), s["kv_len"].tolist(), s["page_table"].tolist()
    pos = torch.cat([torch.arange(length - starts[b + 1] + starts[b], length) for b, length in enumerate(lens)]).cuda()
    q, k = (_turned64(_unit64(s[n], s[n + "_weight"]).transpose(0, 1), s, pos).transpose(0, 1) for n in ("q", "k"))
    k_cache, v_cache = s["k_cache"].double(), s["v_cache"].double()
    scales = [None if x is None else x.double().clone() for x in (s["k_scale"], s["v_scale"])]
    for b, length in enumerate(lens):
        at, t = length - (starts[b + 1] - starts[b]), starts[b]
        while t < starts[b + 1]:
            page, slot = table[b][at // P], at % P
            n = min(P - slot, starts[b + 1] - t)
            for x, cache, scale in ((k, k_cache, scales[0]), (s["v"].double(), v_cache, scales[1])):
                new = x[t:t + n].transpose(0, 1)                                   # [heads, n, d]
                if scale is not None:
                    size = new.abs().amax(dim=(1, 2)).clamp(min=1e-12)
                    fit = torch.exp2(torch.ceil(torch.log2(size / E4M3_MAX)))
                    fit = torch.where(size <= E4M3_MAX * fit / 2, fit / 2, fit)        # the logarithm of an exact power of two may come out above it
                    if slot > 0:
                        fit = torch.maximum(fit, scale[page])
                        cache[page, :, :slot] *= (scale[page] / fit)[:, None, None]
                    scale[page] = fit
                    new = new / fit[:, None, None]
                cache[page, :, slot:slot + n] = new
            t, at = t + n, at + n
    return {"q": q, "k_cache": k_cache, "v_cache": v_cache, "k_scale": scales[0], "v_scale": scales[1]}


def _exact_attend(s):
    c = s["case"]
    H, Hk, d, P = c["heads"], c["kv_heads"], c["dim"], c["page"]
    G = H // Hk
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    starts, lens = s["q_start"].tolist(), s["kv_len"].tolist()
    for b, length in enumerate(lens):
        if length == 0:
            continue
        lo, hi = starts[b], starts[b + 1]
        pages = s["page_table"][b, :-(-length // P)].long()
        rows = torch.tensor(_seen(c, length, hi - lo), device="cuda")
        j = torch.arange(length, device="cuda")
        hidden = (j[None] >= rows[:, 1:2]) | ((j[None] < rows[:, :1]) & (j[None] >= rows[:, 2:]))
        some = rows[:, 1] > 0
        for h in range(Hk):
            def taken(cache, scale):
                x = cache[:, h].view(torch.uint8)[pages].view(torch.float8_e4m3fn).double() if c["fp8"] else cache[:, h][pages].double()
                x = x if scale is None else x * scale[pages, h].double()[:, None, None]
                return x.reshape(-1, d)[:length]
            kk, vv = taken(s["k_cache"], s["k_scale"]), taken(s["v_cache"], s["v_scale"])
            for g in range(G):
                a = s["q"][lo:hi, h * G + g].double() @ kk.T * d ** -0.5
                a[hidden] = -math.inf
                lse[lo:hi, h * G + g] = torch.logsumexp(a, dim=1)
                out[lo:hi, h * G + g][some] = torch.softmax(a[some], dim=1) @ vv
    return {"out": out, "lse": lse}


def _exact_copy(s, src, dst):
    """The pools with page src[i] at dst[i]."""
    got = {}
    for n in ("k_cache", "v_cache", "k_scale", "v_scale"):
        if s[n] is None:
            got[n] = None
            continue
        x = s[n].double()
        if dst:
            x[torch.tensor(dst, device="cuda")] = x[torch.tensor(src, device="cuda")]
        got[n] = x
    return got


def _exact_book(s):
    """The same by hand, entry after entry."""
    c = s["case"]
    op, P = c["op"], c["page"]
    table, refs, held = s["page_table"].tolist(), s["refs"].tolist(), s["kv_len"].tolist()
    more = {}
    src, dst = [], []
    if op == "fork":
        parent = s["parent"].tolist()
        rows = [list(table[p]) if p >= 0 else [-1] * len(table[0]) for p in parent]
        for sign, tables in ((-1, table), (1, rows)):
            for row in tables:
                for e in row:
                    if e >= 0:
                        refs[e] += sign
        table = rows
        more["kv_len"] = torch.tensor([held[p] if p >= 0 else 0 for p in parent])
    elif op == "trim":
        for b, n in enumerate(held):
            lo = (n // c["frame"] - c["window"] + 1) * c["frame"] if c["window"] else 0
            for i, e in enumerate(table[b]):
                if e >= 0 and (i * P >= n or (i * P >= c["sink"] and (i + 1) * P <= lo)):
                    refs[e] -= 1
                    table[b][i] = -1
    elif op == "reserve":
        new = s["kv_new"].tolist()
        free = [p for p, r in enumerate(refs) if r == 0]
        writers = {}
        for b, n in enumerate(held):
            if n % P and new[b] > n and refs[table[b][n // P]] > 1:
                writers.setdefault(table[b][n // P], []).append(b)
        keeps = {w[0] for p, w in writers.items() if len(w) == refs[p]}
        copies = {b for w in writers.values() for b in w} - keeps
        wanted = [(b, i) for b, n in enumerate(held) for i in ([n // P] if b in copies else []) + [i for i in range(-(-n // P), -(-new[b] // P)) if table[b][i] < 0]]
        pairs = [(-1, -1)] * len(held)
        if len(wanted) <= len(free):
            for (b, i), p in zip(wanted, free):
                if table[b][i] >= 0:
                    refs[table[b][i]] -= 1
                    pairs[b] = (table[b][i], p)
                table[b][i] = p
                refs[p] = 1
        src, dst = [p for p, _ in pairs if p >= 0], [p for _, p in pairs if p >= 0]
        more["src"], more["dst"] = torch.tensor([p for p, _ in pairs]), torch.tensor([p for _, p in pairs])
    else:
        used = sum(r > 0 for r in refs)
        src = [p for p, r in enumerate(refs) if r > 0 and p >= used]
        dst = [p for p, r in enumerate(refs) if r == 0 and p < used]
        to = dict(zip(src, dst))
        table = [[to.get(e, e) for e in row] for row in table]
        for p, q in to.items():
            refs[q], refs[p] = refs[p], 0
        pad = [-1] * (len(refs) // 2 - len(src))
        more["src"], more["dst"] = torch.tensor(src + pad), torch.tensor(dst + pad)
    pools = _exact_copy(s, src, dst) if op in ("reserve", "compact") else {}
    return {"page_table": torch.tensor(table), "refs": torch.tensor(refs)} | more | pools


def exact(case, seed):
    s = prepare(case, seed)
    return {"whole": _exact_whole, "append": _exact_append, "attend": _exact_attend}.get(case["op"], _exact_book)(s)
