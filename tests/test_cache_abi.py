"""Host-side checks of the paged cache's calls, without a GPU: the structs match the header, and every argument that the calls do not
serve is refused before anything is enqueued."""
import ctypes
import math
import os
import re

import pytest
import torch

import paper_2609_23153_b200 as sa

FAKE, OFF8, OFF16, NULL = 0x10000, 0x10008, 0x10010, None      # (never dereferenced: every call here is refused)


@pytest.fixture(scope="module")
def lib():
    from paper_2609_23153_b200 import build
    build.build()
    return sa.lib()


def make_call(**change):
    """The two calls' arguments, all of them served, but for what `change` names as "struct.field" or "argument"."""
    s = {
        "cache": sa.CacheShape(ctypes.sizeof(sa.CacheShape), sa.VERSION, sa.FP8_E4M3, 10, 4, 64, 128, 0, 4 * 64 * 128, 64 * 128, 128),
        "batch": sa.Batch(ctypes.sizeof(sa.Batch), sa.VERSION, 2, 6, 3, 5, FAKE, FAKE, NULL),
        "rotary": sa.RotaryShape(ctypes.sizeof(sa.RotaryShape), sa.VERSION, 128, 0, 1000, 1, FAKE, FAKE, NULL, NULL),
        "q": sa.Rows(FAKE, 8 * 128, 128), "k": sa.Rows(FAKE, 4 * 128, 128), "v": sa.Rows(FAKE, 4 * 128, 128), "out": sa.Rows(FAKE, 8 * 128, 128),
    }
    a = dict(H=8, k_cache=FAKE, v_cache=FAKE, k_scale=FAKE, v_scale=FAKE, workspace=FAKE, bytes=1 << 30, frame=1, window=0, scale=0.0, lse=NULL)
    for name, value in change.items():
        if "__" in name:
            struct, field = name.split("__")
            assert hasattr(s[struct], field)
            setattr(s[struct], field, value)
        else:
            assert name in a or name in s
            (s if name in s else a)[name] = value
    return s, a


def ref(x):
    return None if x is None else ctypes.byref(x)


def append(lib, **change):
    s, a = make_call(**change)
    return lib.sparkattn_cache_append(ref(s["cache"]), ref(s["batch"]), ref(s["rotary"]), ref(s["q"]), a["H"], ref(s["k"]), ref(s["v"]), a["k_cache"], a["v_cache"],
                                      a["k_scale"], a["v_scale"], ref(s["out"]), a["workspace"], a["bytes"], None)


def attend(lib, **change):
    s, a = make_call(**change)
    return lib.sparkattn_cache_fwd(ref(s["cache"]), ref(s["batch"]), ref(s["q"]), a["H"], a["k_cache"], a["v_cache"], a["k_scale"], a["v_scale"], a["frame"],
                                   a["window"], a["scale"], ref(s["out"]), a["lse"], a["workspace"], a["bytes"], None)


def test_structs_have_the_headers_sizes():
    # no implicit padding but behind nothing: 8 four-byte fields and 3 strides; 6 and 3 pointers; a pointer and 2 strides; 6 and 4 pointers
    assert [ctypes.sizeof(x) for x in (sa.CacheShape, sa.Batch, sa.Rows, sa.RotaryShape)] == [56, 48, 24, 56]


BOTH = [
    (dict(cache=None), "INVALID_ARG"), (dict(batch=None), "INVALID_ARG"),
    (dict(cache__struct_size=48), "INVALID_ARG"), (dict(cache__version=9), "INVALID_ARG"), (dict(cache__reserved=1), "INVALID_ARG"),
    (dict(batch__struct_size=40), "INVALID_ARG"), (dict(batch__version=0), "INVALID_ARG"),
    (dict(cache__dtype=2), "INVALID_ARG"), (dict(cache__dtype=-1), "INVALID_ARG"),
    (dict(cache__pages=0), "INVALID_ARG"), (dict(cache__H=0), "INVALID_ARG"), (dict(cache__H=-4), "INVALID_ARG"),
    (dict(batch__B=0), "INVALID_ARG"), (dict(batch__T=0), "INVALID_ARG"), (dict(batch__T=-6), "INVALID_ARG"),
    (dict(batch__max_new=0), "INVALID_ARG"), (dict(batch__max_pages=0), "INVALID_ARG"),
    (dict(batch__max_new=7, batch__q_start=FAKE), "INVALID_ARG"),       # more than there are rows
    (dict(batch__max_new=2), "INVALID_ARG"), (dict(batch__T=7), "INVALID_ARG"),      # no starts: T / B rows each
    (dict(cache__d=96), "UNSUPPORTED_SHAPE"), (dict(cache__d=256), "UNSUPPORTED_SHAPE"),
    (dict(cache__page=8), "UNSUPPORTED_SHAPE"), (dict(cache__page=48), "UNSUPPORTED_SHAPE"), (dict(cache__page=256), "UNSUPPORTED_SHAPE"),
    (dict(batch__B=4097, batch__T=3 * 4097), "UNSUPPORTED_SHAPE"), (dict(cache__H=65536), "UNSUPPORTED_SHAPE"),
    (dict(cache__stride_n=64), "INVALID_ARG"), (dict(cache__stride_h=0), "INVALID_ARG"), (dict(cache__stride_page=0), "INVALID_ARG"),
    (dict(cache__stride_n=136), "MISALIGNED"), (dict(cache__stride_h=64 * 128 + 8), "MISALIGNED"), (dict(cache__stride_page=4 * 64 * 128 + 8), "MISALIGNED"),
    (dict(cache__dtype=0, k_scale=NULL, v_scale=NULL, cache__stride_n=132), "MISALIGNED"),
    (dict(k_cache=NULL), "INVALID_ARG"), (dict(v_cache=NULL), "INVALID_ARG"), (dict(workspace=NULL), "INVALID_ARG"),
    (dict(batch__page_table=NULL), "INVALID_ARG"), (dict(batch__kv_len=NULL), "INVALID_ARG"),
    (dict(k_scale=NULL), "INVALID_ARG"), (dict(v_scale=NULL), "INVALID_ARG"),
    (dict(cache__dtype=0), "INVALID_ARG"), (dict(cache__dtype=0, k_scale=NULL), "INVALID_ARG"),      # bf16 pages have no scales
    (dict(k_cache=OFF8), "MISALIGNED"), (dict(v_cache=OFF8), "MISALIGNED"), (dict(workspace=OFF16), "MISALIGNED"),
    (dict(q__data=NULL), "INVALID_ARG"), (dict(out__data=NULL), "INVALID_ARG"), (dict(q__stride_t=-8), "INVALID_ARG"), (dict(q__stride_h=-8), "INVALID_ARG"),
    (dict(out__stride_t=0), "INVALID_ARG"), (dict(out__stride_h=0), "INVALID_ARG"),
    (dict(q__data=OFF8), "MISALIGNED"), (dict(out__data=OFF8), "MISALIGNED"), (dict(q__stride_t=4), "MISALIGNED"), (dict(out__stride_h=132), "MISALIGNED"),
    (dict(H=0), "INVALID_ARG"), (dict(H=-8), "INVALID_ARG"),
    (dict(H=0x7ffffffc), "UNSUPPORTED_SHAPE"),
]


@pytest.mark.parametrize("change,status", BOTH, ids=lambda x: "-".join(x) if isinstance(x, dict) else x)
@pytest.mark.parametrize("call", [append, attend])
def test_refusals_of_both_calls(lib, call, change, status):
    assert call(lib, **change) == getattr(sa, "E_" + status)


@pytest.mark.parametrize("change,status", [
    (dict(q=None), "INVALID_ARG"), (dict(out=None), "INVALID_ARG"),      # queries and where they go: both or neither
    (dict(k=None), "INVALID_ARG"), (dict(v=None), "INVALID_ARG"), (dict(k__data=NULL), "INVALID_ARG"), (dict(v__data=NULL), "INVALID_ARG"),
    (dict(k__data=OFF8), "MISALIGNED"), (dict(v__stride_t=4 * 128 + 4), "MISALIGNED"),
    (dict(rotary__struct_size=0), "INVALID_ARG"), (dict(rotary__version=2), "INVALID_ARG"),
    (dict(rotary__cos=NULL), "INVALID_ARG"), (dict(rotary__sin=NULL), "INVALID_ARG"), (dict(rotary__rows=0), "INVALID_ARG"),
    (dict(rotary__interleaved=2), "INVALID_ARG"), (dict(rotary__axes=0), "INVALID_ARG"), (dict(rotary__axes=5, rotary__positions=FAKE), "INVALID_ARG"),
    (dict(rotary__axes=3), "INVALID_ARG"),                               # several axes without positions
    (dict(rotary__rot=0), "UNSUPPORTED_SHAPE"), (dict(rotary__rot=24), "UNSUPPORTED_SHAPE"), (dict(rotary__rot=144), "UNSUPPORTED_SHAPE"),
    (dict(rotary__rows=1 << 26), "UNSUPPORTED_SHAPE"),                   # 2^32 entries
    (dict(rotary__cos=OFF8), "MISALIGNED"), (dict(rotary__sin=OFF8), "MISALIGNED"),
    (dict(bytes=255), "WORKSPACE_TOO_SMALL"), (dict(bytes=0), "WORKSPACE_TOO_SMALL"),
], ids=lambda x: "-".join(x) if isinstance(x, dict) else x)
def test_refusals_of_append(lib, change, status):
    assert append(lib, **change) == getattr(sa, "E_" + status)


@pytest.mark.parametrize("change,status", [
    (dict(q=None), "INVALID_ARG"), (dict(out=None), "INVALID_ARG"), (dict(H=10), "INVALID_ARG"),
    (dict(frame=-1), "INVALID_ARG"), (dict(window=-1), "INVALID_ARG"), (dict(frame=0, window=1), "INVALID_ARG"),
    (dict(scale=-1.0), "INVALID_ARG"), (dict(scale=math.inf), "INVALID_ARG"), (dict(scale=math.nan), "INVALID_ARG"),
    (dict(bytes=255), "WORKSPACE_TOO_SMALL"), (dict(bytes=0), "WORKSPACE_TOO_SMALL"),
    (dict(cache__H=4096, H=4096, batch__max_pages=1 << 20), "UNSUPPORTED_SHAPE"),      # more key tiles than 31 bits count
], ids=lambda x: "-".join(x) if isinstance(x, dict) else x)
def test_refusals_of_fwd(lib, change, status):
    assert attend(lib, **change) == getattr(sa, "E_" + status)


def test_workspace_of_what_is_refused_is_nothing(lib):
    for change in (dict(cache__d=96), dict(H=10), dict(batch__T=7), dict(cache__version=9)):
        s, a = make_call(**change)
        assert lib.sparkattn_cache_workspace_bytes(ref(s["cache"]), ref(s["batch"]), a["H"]) == 0
    assert lib.sparkattn_cache_workspace_bytes(None, None, 8) == 0


def test_binding_refuses_layouts():
    """What the library cannot see, the binding refuses: ranks, types, strided last dimensions, sizes that differ, tensors on the host."""
    bf16, i32, f32 = torch.bfloat16, torch.int32, torch.float32
    pool, scale = torch.zeros((4, 2, 16, 64), dtype=torch.uint8), torch.ones((4, 2))
    cache = sa.KVCache(pool, pool, scale, scale)
    k, q = torch.zeros((2, 2, 64), dtype=bf16), torch.zeros((2, 4, 64), dtype=bf16)
    table, lens = torch.zeros((1, 3), dtype=i32), torch.full((1,), 5, dtype=i32)
    cos = torch.ones((9, 32))

    def bad_cache(**change):
        return cache._replace(**change)

    pools = [bad_cache(k=pool[0]), bad_cache(v=pool[:, :, :8]), bad_cache(k=pool.transpose(2, 3), v=pool.transpose(2, 3)), bad_cache(v=pool.float()),
             bad_cache(k=pool.float(), v=pool.float()), bad_cache(k_scale=None), bad_cache(v_scale=scale.double()), bad_cache(k_scale=scale[:3]),
             bad_cache(k_scale=scale.t().contiguous().t()), sa.KVCache(pool.to(bf16), pool.to(bf16), scale, scale)]
    calls = [lambda c=c: sa.cache_append(c, k, k, table, lens) for c in pools] + [lambda c=c: sa.cache_fwd(q, c, table, lens) for c in pools]
    for t, n, start in ((table.long(), lens, None), (table[0], lens, None), (table, lens.float(), None), (table, lens.repeat(2), None),
                        (table, lens, torch.zeros(3, dtype=i32)), (table, lens, torch.zeros(2)), (torch.zeros((1, 6), dtype=i32)[:, ::2], lens, None)):
        calls += [lambda t=t, n=n, s=start: sa.cache_append(cache, k, k, t, n, q_start=s), lambda t=t, n=n, s=start: sa.cache_fwd(q, cache, t, n, q_start=s)]
    calls += [lambda: sa.cache_append(cache, k[0], k, table, lens), lambda: sa.cache_append(cache, k, k[:1], table, lens), lambda: sa.cache_append(cache, q, k, table, lens),
              lambda: sa.cache_append(cache, k.float(), k, table, lens), lambda: sa.cache_fwd(q[:, :, ::2], cache, table, lens), lambda: sa.cache_fwd(q.half(), cache, table, lens)]
    for rotary in (sa.Rotary(cos, cos[:8]), sa.Rotary(cos.double(), cos.double()), sa.Rotary(cos[0], cos[0]), sa.Rotary(cos, cos, positions=torch.zeros(3, dtype=i32)),
                   sa.Rotary(cos, cos, positions=torch.zeros(2)), sa.Rotary(cos, cos, axis=torch.zeros(31, dtype=i32)),
                   sa.Rotary(cos, cos, positions=torch.zeros((2, 3), dtype=i32))):
        calls.append(lambda r=rotary: sa.cache_append(cache, k, k, table, lens, rotary=r))
    for call in calls:
        with pytest.raises(ValueError) as e:
            call()
        assert "CUDA" not in str(e.value)
    for call in (lambda: sa.cache_append(cache, k, k, table, lens), lambda: sa.cache_fwd(q, cache, table, lens)):      # all as it should be, but on the host
        with pytest.raises(ValueError, match="CUDA device"):
            call()
    with pytest.raises(TypeError):
        sa.cache_fwd(q, (pool, [1], scale, scale), table, lens)


@pytest.mark.parametrize("page,d", [(16, 64), (128, 128)])
@pytest.mark.parametrize("fp8", [True, False])
def test_alloc_cache(page, d, fp8):
    c = sa.alloc_cache(3, 2, page, d, fp8=fp8, device="cpu")
    assert c.k.shape == c.v.shape == (3, 2, page, d) and c.k.data_ptr() != c.v.data_ptr()
    assert c.k.dtype == (torch.float8_e4m3fn if fp8 else torch.bfloat16)
    assert (c.k_scale is not None and c.k_scale.shape == (3, 2) and c.k_scale.dtype == torch.float32) if fp8 else c.k_scale is None


def test_what_threads_write_into_a_tile_is_fenced_before_the_next_copy():
    """The operand warps put zeros among V's codes, and both kernels marks' zeros among values: ordinary stores where TMA writes next.  Between them and the
    arrival that frees the place stands the fence that orders the two."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    chunk, decode = (re.sub(r"//[^\n]*", "", open(os.path.join(root, "paper_2609_23153_b200", "csrc", f)).read()) for f in ("cache_chunk.cu", "cache_fwd.cu"))
    codes = chunk[chunk.index("convert(sRaw + slot"):]
    assert codes.index("fence.proxy.async") < codes.index("mbar_arrive(raw_free") < codes.index("mbar_arrive(v_full")
    edge = chunk[chunk.index("*chunk = make_uint4"):chunk.index("convert(sRaw + slot")]
    assert re.search(r"if constexpr \(!FP8\) asm volatile\(.fence\.proxy\.async", edge)
    mark = decode[decode.index("mark_tile("):decode.index("cache_decode_kernel(")]
    assert mark.index("mark_word<") < mark.index("fence.proxy.async")


def test_queries_in_parts_are_as_exact_as_the_header_says():
    """Every bf16 of a row whose largest entry lies in [128, 256): as two E4M3 parts exact from 2^-9 of the largest on and off by 2^-17 of it at most
    below, as fp16 from 2^-24 on and by 2^-32."""
    x = torch.arange(1, 0x7f80, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).double()
    x = x[x < 256]
    e4m3 = lambda y: y.float().to(torch.float8_e4m3fn).double()
    high = e4m3(x)
    off = (x - high - e4m3(x - high)).abs()
    assert off.max() == 128 * 2.0 ** -17 and (off[x >= 128 * 2.0 ** -9] == 0).all()
    off = (x - x.float().half().double()).abs()
    assert off.max() == 128 * 2.0 ** -32 and (off[x >= 128 * 2.0 ** -24] == 0).all()
