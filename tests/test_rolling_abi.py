"""Host-side checks of the norm, of attention with first tokens and of the cache's pages, without a GPU: struct sizes, and what the calls refuse."""
import ctypes
import math

import pytest
import torch

import paper_2609_23153_b200 as sa
from test_cache_abi import FAKE, NULL, OFF8, OFF16, make_call, ref

CACHE = 4 * 64 * 128


@pytest.fixture(scope="module")
def lib():
    from paper_2609_23153_b200 import build
    build.build()
    return sa.lib()


def test_structs_have_the_headers_sizes():
    # 5 four-byte fields, a pad and 2 pointers; 6 and 2 pointers
    assert [ctypes.sizeof(x) for x in (sa.NormShape, sa.BookShape)] == [40, 40]


def changed(structs, args, change):
    for name, value in change.items():
        if "__" in name:
            struct, field = name.split("__")
            assert hasattr(structs[struct], field)
            setattr(structs[struct], field, value)
        else:
            assert name in args or name in structs, name
            (structs if name in structs else args)[name] = value
    return structs, args


def norm_shape():
    return sa.NormShape(ctypes.sizeof(sa.NormShape), sa.VERSION, sa.FP32, 0, 1e-6, 0, FAKE, FAKE)


NORMS = [
    (dict(norm__struct_size=32), "INVALID_ARG"), (dict(norm__version=0), "INVALID_ARG"), (dict(norm__pad=1), "INVALID_ARG"),
    (dict(norm__weight_dtype=sa.FP8_E4M3), "INVALID_ARG"), (dict(norm__weight_dtype=3), "INVALID_ARG"), (dict(norm__weight_dtype=-1), "INVALID_ARG"),
    (dict(norm__per_head=2), "INVALID_ARG"), (dict(norm__eps=0.0), "INVALID_ARG"), (dict(norm__eps=-1e-6), "INVALID_ARG"), (dict(norm__eps=1e-39), "INVALID_ARG"),
    (dict(norm__eps=math.inf), "INVALID_ARG"), (dict(norm__eps=math.nan), "INVALID_ARG"), (dict(norm__q_weight=OFF8), "MISALIGNED"), (dict(norm__k_weight=OFF8), "MISALIGNED"),
]


def append_norm(lib, **change):
    s, a = make_call()
    s["norm"] = norm_shape()
    s, a = changed(s, a, change)
    return lib.sparkattn_cache_append_norm(ref(s["cache"]), ref(s["batch"]), ref(s["norm"]), ref(s["rotary"]), ref(s["q"]), a["H"], ref(s["k"]), ref(s["v"]), a["k_cache"],
                                           a["v_cache"], a["k_scale"], a["v_scale"], ref(s["out"]), a["workspace"], a["bytes"], None)


def shape(B=2, H=8, N=100, d=128):
    return sa.Shape(ctypes.sizeof(sa.Shape), sa.VERSION, B, H, N, d, 128 if d == 128 else 64, 0, H * N * d, N * d, d, 0.0, 0)


def norm_rotate(lib, **change):
    s = {"q": shape(), "qo": shape(), "k": shape(H=4), "ko": shape(H=4), "norm": norm_shape(),
         "rotary": sa.RotaryShape(ctypes.sizeof(sa.RotaryShape), sa.VERSION, 128, 0, 1000, 1, FAKE, FAKE, NULL, NULL)}
    a = dict(pq=FAKE, pqo=FAKE, pk=FAKE, pko=FAKE, workspace=FAKE, bytes=256)
    s, a = changed(s, a, change)
    return lib.sparkattn_norm_rotate(ref(s["q"]), a["pq"], ref(s["qo"]), a["pqo"], ref(s["k"]), a["pk"], ref(s["ko"]), a["pko"], ref(s["norm"]), ref(s["rotary"]),
                                     a["workspace"], a["bytes"], None)


@pytest.mark.parametrize("change,status", NORMS, ids=lambda x: "-".join(x) if isinstance(x, dict) else x)
@pytest.mark.parametrize("call", [append_norm, norm_rotate])
def test_norms_that_are_refused(lib, call, change, status):
    assert call(lib, **change) == getattr(sa, "E_" + status)


@pytest.mark.parametrize("change,status", [
    (dict(norm=None, rotary=None), "INVALID_ARG"),
    (dict(q=None), "INVALID_ARG"), (dict(qo=None), "INVALID_ARG"), (dict(k=None), "INVALID_ARG"), (dict(ko=None), "INVALID_ARG"),
    (dict(pq=NULL), "INVALID_ARG"), (dict(pqo=NULL), "INVALID_ARG"), (dict(pk=NULL), "INVALID_ARG"), (dict(pko=NULL), "INVALID_ARG"), (dict(workspace=NULL), "INVALID_ARG"),
    (dict(q__B=1), "INVALID_ARG"), (dict(k__N=99), "INVALID_ARG"), (dict(qo__H=4), "INVALID_ARG"), (dict(k=shape(B=3, H=4), ko=shape(B=3, H=4)), "INVALID_ARG"),
    (dict(k=shape(H=4, N=99), ko=shape(H=4, N=99)), "INVALID_ARG"), (dict(k=shape(H=4, d=64), ko=shape(H=4, d=64)), "INVALID_ARG"),
    (dict(q__d=96), "UNSUPPORTED_SHAPE"), (dict(qo__stride_n=132), "MISALIGNED"), (dict(k__stride_h=100 * 128 + 8), "MISALIGNED"),
    (dict(q__N=0), "INVALID_ARG"), (dict(qo__stride_n=64), "INVALID_ARG"),
    (dict(pq=OFF8), "MISALIGNED"), (dict(pko=OFF8), "MISALIGNED"), (dict(workspace=OFF16), "MISALIGNED"), (dict(bytes=255), "WORKSPACE_TOO_SMALL"),
    (dict(rotary__rot=144), "UNSUPPORTED_SHAPE"), (dict(rotary__axes=2), "INVALID_ARG"), (dict(rotary__cos=OFF8), "MISALIGNED"),
], ids=lambda x: "-".join(x) if isinstance(x, dict) else x)
def test_refusals_of_norm_rotate(lib, change, status):
    assert norm_rotate(lib, **change) == getattr(sa, "E_" + status)


@pytest.mark.parametrize("change,status", [
    (dict(sink=-1), "INVALID_ARG"), (dict(frame=0, window=1), "INVALID_ARG"), (dict(window=-1), "INVALID_ARG"), (dict(q=None), "INVALID_ARG"), (dict(H=10), "INVALID_ARG"),
    (dict(scale=math.nan), "INVALID_ARG"), (dict(bytes=255), "WORKSPACE_TOO_SMALL"), (dict(k_cache=OFF8), "MISALIGNED"),
], ids=lambda x: "-".join(x) if isinstance(x, dict) else x)
def test_refusals_of_attention_with_first_tokens(lib, change, status):
    s, a = make_call()
    a["sink"] = 4
    s, a = changed(s, a, change)
    assert lib.sparkattn_cache_fwd_sink(ref(s["cache"]), ref(s["batch"]), ref(s["q"]), a["H"], a["k_cache"], a["v_cache"], a["k_scale"], a["v_scale"], a["frame"],
                                        a["window"], a["sink"], a["scale"], ref(s["out"]), a["lse"], a["workspace"], a["bytes"], None) == getattr(sa, "E_" + status)


def book_call(lib, name, **change):
    s = {"book": sa.BookShape(ctypes.sizeof(sa.BookShape), sa.VERSION, 3, 20, 50, 64, FAKE, FAKE)}
    a = dict(kv_len=FAKE, parent=FAKE, B_out=3, kv_new=FAKE, table_out=FAKE + 4096, len_out=FAKE + 4096, refs_out=FAKE, src=FAKE, dst=FAKE, frame=1, window=0, sink=0,
             workspace=FAKE, bytes=512)
    s, a = changed(s, a, change)
    args = dict(fork=("kv_len", "parent", "B_out", "table_out", "len_out", "refs_out"), reserve=("kv_len", "kv_new", "table_out", "refs_out", "src", "dst"),
                trim=("kv_len", "frame", "window", "sink", "table_out", "refs_out"), compact=("table_out", "refs_out", "src", "dst"))[name]
    return getattr(lib, "sparkattn_pages_" + name)(ref(s["book"]), *(a[x] for x in args), a["workspace"], a["bytes"], None)


BOOKS = [
    (dict(book=None), "INVALID_ARG"), (dict(book__struct_size=32), "INVALID_ARG"), (dict(book__version=7), "INVALID_ARG"),
    (dict(book__B=0), "INVALID_ARG"), (dict(book__max_pages=0), "INVALID_ARG"), (dict(book__pages=0), "INVALID_ARG"), (dict(book__pages=-5), "INVALID_ARG"),
    (dict(book__B=4097), "UNSUPPORTED_SHAPE"), (dict(book__max_pages=1 << 30), "UNSUPPORTED_SHAPE"), (dict(book__pages=(1 << 30) + 1), "UNSUPPORTED_SHAPE"),
    (dict(book__page=8), "UNSUPPORTED_SHAPE"), (dict(book__page=48), "UNSUPPORTED_SHAPE"),
    (dict(book__page_table=NULL), "INVALID_ARG"), (dict(book__refs=NULL), "INVALID_ARG"), (dict(table_out=NULL), "INVALID_ARG"), (dict(refs_out=NULL), "INVALID_ARG"),
    (dict(workspace=NULL), "INVALID_ARG"), (dict(workspace=OFF16), "MISALIGNED"), (dict(bytes=511), "WORKSPACE_TOO_SMALL"),
]
ONES = [
    ("fork", dict(kv_len=NULL), "INVALID_ARG"), ("fork", dict(parent=NULL), "INVALID_ARG"), ("fork", dict(len_out=NULL), "INVALID_ARG"), ("fork", dict(B_out=0), "INVALID_ARG"),
    ("fork", dict(B_out=4097), "UNSUPPORTED_SHAPE"), ("fork", dict(table_out=FAKE), "INVALID_ARG"), ("fork", dict(len_out=FAKE), "INVALID_ARG"),      # in place
    ("reserve", dict(kv_len=NULL), "INVALID_ARG"), ("reserve", dict(kv_new=NULL), "INVALID_ARG"), ("reserve", dict(src=NULL), "INVALID_ARG"), ("reserve", dict(dst=NULL), "INVALID_ARG"),
    ("trim", dict(kv_len=NULL), "INVALID_ARG"), ("trim", dict(frame=-1), "INVALID_ARG"), ("trim", dict(window=-1), "INVALID_ARG"), ("trim", dict(sink=-1), "INVALID_ARG"),
    ("trim", dict(frame=0, window=2), "INVALID_ARG"), ("compact", dict(src=NULL), "INVALID_ARG"), ("compact", dict(dst=NULL), "INVALID_ARG"),
]


@pytest.mark.parametrize("name,change,status", [(n, c, s) for n in ("fork", "reserve", "trim", "compact") for c, s in BOOKS] + ONES,
                         ids=lambda x: "-".join(x) if isinstance(x, dict) else x)
def test_refusals_of_books(lib, name, change, status):
    assert book_call(lib, name, **change) == getattr(sa, "E_" + status)


def test_workspace_of_books(lib):
    book = sa.BookShape(ctypes.sizeof(sa.BookShape), sa.VERSION, 3, 20, 50, 64, FAKE, FAKE)
    assert lib.sparkattn_pages_workspace_bytes(ctypes.byref(book)) == 512
    book.pages = 1000
    assert lib.sparkattn_pages_workspace_bytes(ctypes.byref(book)) == 256 + 4096
    book.page = 17
    assert lib.sparkattn_pages_workspace_bytes(ctypes.byref(book)) == 0 == lib.sparkattn_pages_workspace_bytes(None)


@pytest.mark.parametrize("change,status", [
    (dict(a=None), "INVALID_ARG"), (dict(b=None), "INVALID_ARG"), (dict(a__d=96), "UNSUPPORTED_SHAPE"), (dict(b__page=8), "UNSUPPORTED_SHAPE"), (dict(a__reserved=1), "INVALID_ARG"),
    (dict(k_a=NULL), "INVALID_ARG"), (dict(v_b=NULL), "INVALID_ARG"), (dict(ks_a=NULL), "INVALID_ARG"), (dict(vs_b=NULL), "INVALID_ARG"), (dict(a__dtype=0), "INVALID_ARG"),
    (dict(k_a=OFF8), "MISALIGNED"), (dict(v_b=OFF8), "MISALIGNED"), (dict(b__stride_n=136), "MISALIGNED"),
    (dict(b__H=5), "INVALID_ARG"), (dict(b__page=32), "INVALID_ARG"), (dict(b__d=64), "INVALID_ARG"),
    (dict(b=sa.CacheShape(ctypes.sizeof(sa.CacheShape), sa.VERSION, 0, 10, 4, 64, 128, 0, CACHE, 64 * 128, 128), ks_b=NULL, vs_b=NULL), "INVALID_ARG"),      # another type
    (dict(b__pages=11, k_b=FAKE, v_b=FAKE, ks_b=FAKE, vs_b=FAKE), "INVALID_ARG"),                # the same pool under another struct
    (dict(k_b=FAKE), "INVALID_ARG"), (dict(v_b=FAKE), "INVALID_ARG"), (dict(ks_b=FAKE), "INVALID_ARG"), (dict(vs_b=FAKE), "INVALID_ARG"),      # one of two pools' parts
    (dict(n=-1), "INVALID_ARG"), (dict(src=NULL), "INVALID_ARG"), (dict(dst=NULL), "INVALID_ARG"), (dict(workspace=NULL), "INVALID_ARG"),
    (dict(workspace=OFF16), "MISALIGNED"), (dict(bytes=255), "WORKSPACE_TOO_SMALL"),
], ids=lambda x: "-".join(x) if isinstance(x, dict) else x)
def test_refusals_of_copy_pages(lib, change, status):
    other = FAKE + (1 << 20)
    s = {x: sa.CacheShape(ctypes.sizeof(sa.CacheShape), sa.VERSION, sa.FP8_E4M3, 10, 4, 64, 128, 0, CACHE, 64 * 128, 128) for x in "ab"}
    a = dict(k_a=FAKE, v_a=FAKE, ks_a=FAKE, vs_a=FAKE, k_b=other, v_b=other, ks_b=other, vs_b=other, src=FAKE, dst=FAKE, n=3, workspace=FAKE, bytes=256)
    s, a = changed(s, a, change)
    assert lib.sparkattn_cache_copy_pages(ref(s["a"]), a["k_a"], a["v_a"], a["ks_a"], a["vs_a"], ref(s["b"]), a["k_b"], a["v_b"], a["ks_b"], a["vs_b"], a["src"], a["dst"],
                                          a["n"], a["workspace"], a["bytes"], None) == getattr(sa, "E_" + status)


def test_out_of_pages_has_a_text(lib):
    assert "pages" in sa.status_string(sa.E_OUT_OF_PAGES)


def test_binding_refuses_layouts():
    bf16, i32 = torch.bfloat16, torch.int32
    x = torch.zeros((1, 2, 8, 64), dtype=bf16)
    cos = torch.ones((8, 16))
    w = torch.ones(64)
    norm = sa.Norm(w, w)
    rotate = [dict(q=x[0]), dict(q=x.float()), dict(q=x.transpose(2, 3)), dict(q=x, k=x.half()), dict(q=x, k_out=x), dict(q=x, q_out=x.float()),
              dict(q=x, norm=sa.Norm(w, w.to(bf16))), dict(q=x, norm=sa.Norm(w.half())), dict(q=x, norm=sa.Norm(w[:32])), dict(q=x, norm=sa.Norm(torch.ones(128)[::2])),
              dict(q=x, norm=sa.Norm(torch.ones((3, 64)))), dict(q=x, k=x, norm=sa.Norm(torch.ones((2, 64)), w)), dict(q=x, norm=sa.Norm(torch.ones((1, 2, 64)))),
              dict(q=x, rotary=sa.Rotary(cos, cos[:4])), dict(q=x, rotary=sa.Rotary(cos, cos, positions=torch.zeros(7, dtype=i32))),
              dict(q=x, rotary=sa.Rotary(cos, cos, positions=torch.zeros((8, 2), dtype=i32)))]
    calls = [lambda kw=kw: sa.norm_rotate(**dict(dict(norm=norm), **kw)) for kw in rotate]
    table, lens, refs = torch.zeros((2, 3), dtype=i32), torch.ones(2, dtype=i32), torch.zeros(9, dtype=i32)
    for t, n, r in ((table.long(), lens, refs), (table[0], lens, refs), (torch.zeros((2, 6), dtype=i32)[:, ::2], lens, refs), (table, lens[:1], refs), (table, lens.float(), refs),
                    (table, lens, refs.long()), (table, lens, refs.view(3, 3)), (table, lens, torch.zeros(18, dtype=i32)[::2])):
        calls += [lambda t=t, n=n, r=r: sa.pages_fork(t, n, r, lens), lambda t=t, n=n, r=r: sa.pages_reserve(t, n, r, lens, 16), lambda t=t, n=n, r=r: sa.pages_trim(t, n, r, 16)]
        if n is lens:
            calls.append(lambda t=t, r=r: sa.pages_compact(t, r))
    calls += [lambda: sa.pages_fork(table, lens, refs, lens.long()), lambda: sa.pages_fork(table, lens, refs, table), lambda: sa.pages_reserve(table, lens, refs, lens[:1], 16)]
    pool, scale = torch.zeros((4, 2, 16, 64), dtype=torch.uint8), torch.ones((4, 2))
    cache = sa.KVCache(pool, pool.clone(), scale, scale.clone())
    calls += [lambda: sa.cache_copy_pages(cache, lens.long(), lens), lambda: sa.cache_copy_pages(cache, lens, lens[:1]), lambda: sa.cache_copy_pages(cache, table, table),
              lambda: sa.cache_copy_pages(cache._replace(k_scale=None), lens, lens), lambda: sa.cache_copy_pages(cache, lens, lens, to=cache._replace(k=pool.float()))]
    rows, pages = torch.zeros((2, 2, 64), dtype=bf16), torch.zeros((1, 3), dtype=i32)
    five = torch.full((1,), 5, dtype=i32)
    calls += [lambda: sa.cache_append(cache, rows, rows, pages, five, norm=sa.Norm(w[:32])), lambda: sa.cache_append(cache, rows, rows, pages, five, norm=sa.Norm(None, torch.ones((3, 64))))]
    for i, call in enumerate(calls):
        with pytest.raises(ValueError) as e:
            call()
        assert "CUDA" not in str(e.value), i
    for call in (lambda: sa.norm_rotate(x, x, norm=norm), lambda: sa.pages_fork(table, lens, refs, lens), lambda: sa.pages_reserve(table, lens, refs, lens, 16),
                 lambda: sa.pages_trim(table, lens, refs, 16), lambda: sa.pages_compact(table, refs), lambda: sa.cache_copy_pages(cache, lens, lens),
                 lambda: sa.cache_append(cache, rows, rows, pages, five, norm=norm), lambda: sa.cache_fwd(rows, cache, pages, five, window=3, sink=2)):
        with pytest.raises(ValueError, match="CUDA device"):      # all as it should be, but on the host
            call()
