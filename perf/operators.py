"""The work of the paged key/value cache, as cases that can be timed and compared.

An auto-regressive generator (frames of a video one after another, or the tokens of a text) keeps the keys and values of
what it has made so far in pages of a fixed number of tokens, and does two things with them in every layer of every step:

  append   rotates the new tokens' queries and keys by their positions and writes keys and values into the cache:
           bf16, or E4M3 with one scale per page and head
  attend   softmax attention of the new tokens' queries over the cache: one token (decoding), a few (verifying drafted
           tokens), or a whole prompt or frame at a time, causal by token or by frame

A batch is ragged: sequence b owns the tokens q_start[b] .. q_start[b+1] - 1 of the call and kv_len[b] tokens of the cache,
the new ones included.  Lengths follow from the case alone, values, page order and rotary phases from the seed.

`run` computes the operators with this package's calls where `own` is true, and else with elementary torch operations in
32 bits.
"""
import math

import torch

own = False

E4M3_MAX = 448.0
FRAME_480P = (30, 52)        # latent grid of a 480 x 832 frame: 1560 tokens
LARGEST_FLOPS = 1.0e12
LARGEST_BYTES = 6.5e8


def listed():
    def append(name, batch, old, new, heads, kv_heads, page, fp8, **more):
        return dict(name=name, op="append", batch=batch, old=old, new=new, ragged=False, heads=heads, kv_heads=kv_heads, dim=128, rot=128,
                    page=page, fp8=fp8, axes=1, interleaved=False) | more

    def attend(name, batch, length, new, heads, kv_heads, page, fp8, **more):
        return dict(name=name, op="attend", batch=batch, length=length, new=new, ragged=False, hole=False, heads=heads, kv_heads=kv_heads,
                    dim=128, page=page, fp8=fp8, frame=1, window=0) | more

    return [
        # one conversation, one token: nothing but latency
        append("append_one", 1, 1000, 1, 32, 8, 64, True),
        # a serving step: a token for each of many sequences, the last pages partly filled
        append("append_step", 128, 2047, 1, 40, 8, 16, True, ragged=True),
        # three latent frames at 480P enter the cache of the 1.3B model's layer, rotated by (t, y, x)
        append("append_frames", 1, 9360, 4680, 12, 12, 128, True, axes=3, interleaved=True),
        # prompts of odd lengths into a bf16 cache, half the channels rotated
        append("append_prompts", 8, 300, 4001, 32, 8, 64, False, ragged=True, rot=64),
        # one conversation, one token, a thousand keys: latency again
        attend("decode_one", 1, 1001, 1, 32, 8, 64, True),
        # a serving step over sequences of very different lengths
        attend("decode_step", 64, 8191, 1, 40, 8, 64, True, ragged=True),
        # one long document: few heads, all parallelism has to come from the length
        attend("decode_long", 1, 131071, 1, 32, 8, 128, True),
        # bf16 cache, every head with keys of its own
        attend("decode_bf16", 16, 4095, 1, 12, 12, 32, False, ragged=True),
        # small heads, small pages, a sliding window of a thousand keys
        attend("decode_window", 32, 8000, 1, 16, 4, 16, True, dim=64, ragged=True, window=1000),
        # five drafted tokens of each sequence are verified at once
        attend("verify_step", 8, 16383, 5, 64, 8, 64, True, ragged=True),
        # three latent frames at 480P attend to all earlier ones and to each other's whole frame
        attend("frames", 1, 32760, 4680, 12, 12, 128, True, frame=1560),
        # a piece of each of four prompts, causal by token, behind what is cached already
        attend("prompts", 4, 8000, 2048, 32, 8, 64, True, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kv_heads = rng.choice((1, 2, 4, 8, 12))
        c = dict(op=rng.choice(("append", "attend", "attend")), batch=_log_int(rng, 1, 128), ragged=rng.random() < 0.6, heads=0, kv_heads=kv_heads,
                 dim=rng.choice((64, 128, 128)), page=rng.choice((16, 32, 64, 128)), fp8=rng.random() < 0.7)
        c["heads"] = kv_heads * rng.choice((1, 1, 2, 3, 4, 5, 7, 8, 12, 16))
        if c["heads"] > 64:
            continue
        if c["op"] == "append":
            frames = rng.random() < 0.3
            c.update(old=rng.choice((0, _log_int(rng, 1, 4000))), new=1 if rng.random() < 0.4 else _log_int(rng, 2, 6000),
                     rot=rng.choice((c["dim"], c["dim"] // 2)), axes=3 if frames else 1, interleaved=frames or rng.random() < 0.3)
        else:
            kind = rng.random()
            new = 1 if kind < 0.5 else rng.randint(2, 16) if kind < 0.65 else _log_int(rng, 17, 4700)
            frame = 1 if kind < 0.65 or rng.random() < 0.5 else rng.choice((0, _log_int(rng, 16, 1560)))
            length = new + _log_int(rng, 1, 131072)
            window = 0 if frame == 0 or rng.random() < 0.7 else max(1, _log_int(rng, 1, 2 * length) // frame)
            c.update(length=length, new=new, hole=c["batch"] > 1 and rng.random() < 0.2, frame=frame, window=window)
            if c["batch"] * c["heads"] * new * length > 2.0e9 or c["batch"] * length * c["kv_heads"] * c["dim"] > 4.0e8:
                continue
        w = work(c)
        if w["flops"] <= LARGEST_FLOPS and w["bytes"] <= LARGEST_BYTES:
            return c


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


def _visible(case, length, new):
    """[first, last) of the keys that each new token of a sequence attends to."""
    g, w, rows = case["frame"], case["window"], []
    for pos in range(length - new, length):
        if g == 0:
            rows.append((0, length))
        elif pos < 0:
            rows.append((0, 0))
        else:
            rows.append((max(0, (pos // g - w + 1) * g) if w else 0, min(length, (pos // g + 1) * g)))
    return rows


def work(case):
    lens = _lengths(case)
    T, H, Hk, d = sum(n for _, n in lens), case["heads"], case["kv_heads"], case["dim"]
    size = 1 if case["fp8"] else 2
    pages = sum(-(-length // case["page"]) for length, _ in lens)
    if case["op"] == "append":
        positions = max(length for length, _ in lens) if case["axes"] == 1 else T
        touched = sum((length - 1) // case["page"] - (length - n) // case["page"] + 1 for length, n in lens)
        moved = T * d * (2 * 2 * H + 2 * 2 * Hk + 2 * size * Hk)                   # q read and written, k and v read, cache written
        moved += min(T, positions) * case["rot"] * 4 + 4 * T * case["axes"] + 4 * touched * (1 + (2 * Hk if case["fp8"] else 0))
        return {"bytes": moved, "flops": 3 * T * case["rot"] * (H + Hk)}
    pairs = keys = 0
    for length, n in lens:
        rows = _visible(case, length, n)
        pairs += sum(hi - lo for lo, hi in rows)
        keys += max((hi for _, hi in rows), default=0) - min((lo for lo, hi in rows if hi > lo), default=0)
    moved = keys * Hk * 2 * d * size + T * H * (2 * 2 * d + 4) + 4 * pages + (8 * pages * Hk if case["fp8"] else 0)
    return {"bytes": moved, "flops": 4 * d * H * pairs}


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


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    lens = _lengths(case)
    B, H, Hk, d, P = case["batch"], case["heads"], case["kv_heads"], case["dim"], case["page"]
    dev = "cuda"
    starts = [0]
    for _, n in lens:
        starts.append(starts[-1] + n)
    T = starts[-1]
    need = [-(-length // P) for length, _ in lens]
    pages = sum(need) + 3
    columns = max(need) + 1
    order = torch.randperm(pages, generator=gen, device=dev).int()
    table = torch.zeros((B, columns), dtype=torch.int32)
    at = 0
    rows = order.cpu()
    for b, n in enumerate(need):
        table[b, :n] = rows[at:at + n]
        at += n
    s = {"case": dict(case), "k_cache": None, "v_cache": None, "k_scale": None, "v_scale": None,
         "page_table": table.to(dev), "kv_len": torch.tensor([length for length, _ in lens], dtype=torch.int32, device=dev),
         "q_start": torch.tensor(starts, dtype=torch.int32, device=dev), "max_new": max(n for _, n in lens)}
    s["k_cache"], s["k_scale"] = _filled((pages, Hk, P, d), case["fp8"], gen)
    s["v_cache"], s["v_scale"] = _filled((pages, Hk, P, d), case["fp8"], gen)
    s["q"] = (1.5 * torch.randn((T, H, d), generator=gen, device=dev)).bfloat16()
    if case["op"] == "append":
        s["k"] = (1.5 * torch.randn((T, Hk, d), generator=gen, device=dev)).bfloat16()
        s["v"] = (1.5 * torch.randn((T, Hk, d), generator=gen, device=dev)).bfloat16()
        pairs = case["rot"] // 2
        longest = max(length for length, _ in lens)
        phase = torch.rand((), generator=gen, device=dev).double()
        if case["axes"] == 3:        # thirds of the pairs turn with t, y and x of the token on the latent grid
            third = -(-pairs // 3)
            axis = torch.tensor([min(m // third, 2) for m in range(pairs)], dtype=torch.int32)
            freq = torch.tensor([10000.0 ** (-(m % third) / third) for m in range(pairs)], dtype=torch.float64)
            n = torch.cat([torch.arange(length - new, length) for length, new in lens])
            hg, wg = FRAME_480P
            s["positions"] = torch.stack([n // (hg * wg), n // wg % hg, n % wg], dim=1).int().to(dev)
            s["axis"] = axis.to(dev)
            rows = max(int(s["positions"].max()) + 1, 64)
        else:
            freq = torch.tensor([10000.0 ** (-m / pairs) for m in range(pairs)], dtype=torch.float64)
            s["positions"] = s["axis"] = None
            rows = longest
        angle = torch.arange(rows, device=dev)[:, None].double() * freq.to(dev)[None] + phase
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
    return s


# --------------------------------------------------------------------------------------------------------------- plain forms

def _owners(s):
    """(sequence, position in it) of every token of the call."""
    T = s["q"].shape[0]
    token = torch.arange(T, device="cuda")
    seq = torch.searchsorted(s["q_start"][1:].long(), token, right=True)
    start, stop = s["q_start"].long()[seq], s["q_start"].long()[seq + 1]
    return seq, s["kv_len"].long()[seq] - (stop - token)


def _rotate(x, cos, sin, interleaved):
    """x [T, heads, d] with the first 2 * cos.shape[-1] channels turned by the angles of cos, sin [T, pairs]."""
    rot = 2 * cos.shape[-1]
    c, n = cos[:, None], sin[:, None]
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * c - b * n, a * n + b * c], dim=-1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * c - b * n, a * n + b * c], dim=-1)
    return torch.cat([turned, x[..., rot:]], dim=-1)


def _phases(s, pos):
    if s["positions"] is None:
        return s["cos"][pos], s["sin"][pos]
    at = s["positions"].long()[:, s["axis"].long()]                # [T, pairs]
    return s["cos"].gather(0, at), s["sin"].gather(0, at)


def _e4m3(x):
    return x.clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).view(torch.uint8)


def _store_fp8(s, x, cache, scale, page, slot):
    """x [T, heads, d] into an E4M3 cache: a page's scale only grows while it fills, and what it holds is encoded again then."""
    P = s["case"]["page"]
    bytes_ = cache.view(torch.uint8)
    size = torch.where(torch.isfinite(x), x.abs(), 0.0).amax(-1)
    fresh = _power_scale(torch.zeros_like(scale).index_reduce_(0, page, size, "amax"))
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
    cos, sin = _phases(s, pos)
    k, v = _rotate(s["k"].float(), cos, sin, c["interleaved"]), s["v"].float()
    page, slot = s["page_table"].long()[seq, pos // c["page"]], pos % c["page"]
    if c["fp8"]:
        _store_fp8(s, k, s["k_cache"], s["k_scale"], page, slot)
        _store_fp8(s, v, s["v_cache"], s["v_scale"], page, slot)
    else:
        s["k_cache"][page, :, slot] = k.bfloat16()
        s["v_cache"][page, :, slot] = v.bfloat16()
    return _rotate(s["q"].float(), cos, sin, c["interleaved"]).bfloat16()


def _plain_attend(s):
    c = s["case"]
    B, n, H, Hk, d = c["batch"], s["max_new"], c["heads"], c["kv_heads"], c["dim"]
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
    seen = key < length[:, None, None]
    if c["frame"] > 0:
        frame = torch.div(pos, c["frame"], rounding_mode="floor")
        seen = seen & (key < (frame + 1) * c["frame"]) & (pos >= 0)
        if c["window"] > 0:
            seen = seen & (key >= (frame - c["window"] + 1) * c["frame"])
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
    return out.bfloat16(), lse.permute(0, 3, 1, 2).reshape(B, n, H)[seq, row]


# ------------------------------------------------------------------------------------------------------------------- passes

def run(s):
    c = s["case"]
    if own:
        import paper_2609_23153_b200 as sa
        cache = sa.KVCache(s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"])
        batch = dict(q_start=s["q_start"], max_new=s["max_new"])
        if c["op"] == "append":
            rotary = sa.Rotary(s["cos"], s["sin"], positions=s["positions"], axis=s["axis"], interleaved=c["interleaved"])
            q = sa.cache_append(cache, s["k"], s["v"], s["page_table"], s["kv_len"], q=s["q"], rotary=rotary, **batch)
        else:
            out, lse = sa.cache_fwd(s["q"], cache, s["page_table"], s["kv_len"], frame_tokens=c["frame"], window=c["window"],
                                    return_lse=True, **batch)
    elif c["op"] == "append":
        q = _plain_append(s)
    else:
        out, lse = _plain_attend(s)
    if c["op"] == "append":
        return {"q": q, "k_cache": s["k_cache"], "v_cache": s["v_cache"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}
    return {"out": out, "lse": lse}


# ------------------------------------------------------------------------------------------------------------ in 64 bits

def _turned64(x, s, t, pos):
    """Heads x [heads, d] of token t at position pos, in 64 bits."""
    c = s["case"]
    pairs = c["rot"] // 2
    m = torch.arange(pairs, device="cuda")
    p = torch.full_like(m, pos) if s["positions"] is None else s["positions"][t].long()[s["axis"].long()]
    w = torch.complex(s["cos"][p, m].double(), s["sin"][p, m].double())
    first, second = (2 * m, 2 * m + 1) if c["interleaved"] else (m, m + pairs)
    z = torch.complex(x[:, first].double(), x[:, second].double()) * w
    y = x.double().clone()
    y[:, first], y[:, second] = z.real, z.imag
    return y


def _exact_append(s):
    c = s["case"]
    P = c["page"]
    q = torch.empty_like(s["q"], dtype=torch.float64)
    k_cache, v_cache = s["k_cache"].double(), s["v_cache"].double()
    scales = [None if x is None else x.double().clone() for x in (s["k_scale"], s["v_scale"])]
    starts, lens, table = s["q_start"].tolist(), s["kv_len"].tolist(), s["page_table"].tolist()
    k = torch.empty_like(s["k"], dtype=torch.float64)
    for b, length in enumerate(lens):
        for t in range(starts[b], starts[b + 1]):
            pos = length - starts[b + 1] + t
            q[t], k[t] = _turned64(s["q"][t], s, t, pos), _turned64(s["k"][t], s, t, pos)
        pos = length - (starts[b + 1] - starts[b])
        t = starts[b]
        while t < starts[b + 1]:
            page, slot = table[b][pos // P], pos % P
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
            t, pos = t + n, pos + n
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
        rows = torch.tensor(_visible(c, length, hi - lo), device="cuda")
        j = torch.arange(length, device="cuda")
        for h in range(Hk):
            def taken(cache, scale):
                x = cache[:, h].view(torch.uint8)[pages].view(torch.float8_e4m3fn).double() if c["fp8"] else cache[:, h][pages].double()
                x = x if scale is None else x * scale[pages, h].double()[:, None, None]
                return x.reshape(-1, d)[:length]
            kk, vv = taken(s["k_cache"], s["k_scale"]), taken(s["v_cache"], s["v_scale"])
            for g in range(G):
                a = s["q"][lo:hi, h * G + g].double() @ kk.T * d ** -0.5
                a[(j[None] < rows[:, :1]) | (j[None] >= rows[:, 1:])] = -math.inf
                some = rows[:, 1] > rows[:, 0]
                lse[lo:hi, h * G + g] = torch.logsumexp(a, dim=1)
                out[lo:hi, h * G + g][some] = torch.softmax(a[some], dim=1) @ vv
    return {"out": out, "lse": lse}


def exact(case, seed):
    lens = _lengths(case)
    if case["op"] == "append":
        if sum(n for _, n in lens) > 20000:        # token by token
            return None
        return _exact_append(prepare(case, seed))
    return _exact_attend(prepare(case, seed))
