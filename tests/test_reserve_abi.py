"""Host-side checks of the reservation that leaves the step's lengths, without a GPU: what it refuses."""
import pytest
import torch

import paper_2609_23153_b200 as sa
from test_cache_abi import FAKE, NULL, ref
from test_rolling_abi import BOOKS, ONES, changed, lib  # noqa: F401  (lib: the fixture)

import ctypes


def reserve_len(lib, **change):
    s = {"book": sa.BookShape(ctypes.sizeof(sa.BookShape), sa.VERSION, 3, 20, 50, 64, FAKE, FAKE)}
    a = dict(kv_len=FAKE, kv_new=FAKE + 4096, kv_len_out=FAKE + 8192, table_out=FAKE + 4096, refs_out=FAKE, src=FAKE, dst=FAKE, workspace=FAKE, bytes=512)
    s, a = changed(s, a, change)
    return lib.sparkattn_pages_reserve_len(ref(s["book"]), *(a[x] for x in ("kv_len", "kv_new", "kv_len_out", "table_out", "refs_out", "src", "dst")), a["workspace"],
                                           a["bytes"], None)


@pytest.mark.parametrize("change,status", BOOKS + [(c, s) for n, c, s in ONES if n == "reserve"] +
                         [(dict(kv_len_out=NULL), "INVALID_ARG"), (dict(kv_len_out=FAKE), "INVALID_ARG"), (dict(kv_len_out=FAKE + 4096), "INVALID_ARG")],
                         ids=lambda x: "-".join(x) if isinstance(x, dict) else x)
def test_refusals(lib, change, status):  # noqa: F811
    assert reserve_len(lib, **change) == getattr(sa, "E_" + status)


def test_binding_refuses_lengths():
    i32 = torch.int32
    table, lens, refs = torch.zeros((2, 3), dtype=i32), torch.ones(2, dtype=i32), torch.zeros(9, dtype=i32)
    for out in (lens.long(), lens[:1], torch.ones(4, dtype=i32)[::2], table[:, :2].contiguous()):
        with pytest.raises(ValueError, match="kv_len_out"):
            sa.pages_reserve(table, lens, refs, lens, 16, kv_len_out=out)
    with pytest.raises(ValueError, match="CUDA device"):
        sa.pages_reserve(table, lens, refs, lens, 16, kv_len_out=torch.ones(2, dtype=i32))
