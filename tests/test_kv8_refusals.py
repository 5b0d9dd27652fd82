"""Refusals of the paged 8-bit KV cache, on the host: every one is made before anything is launched, so none needs a GPU.  Addresses are
numbers that are never followed."""
import ctypes

import pytest
import torch

import paper_2504_19874_b200 as tq
from paper_2504_19874_b200 import build as tq_build

INVALID, UNSUPPORTED, ALIGNMENT, WORKSPACE = 1, 2, 3, 7
A = 1 << 20                                   # an address


@pytest.fixture(scope="module", autouse=True)
def built():
    tq_build.build()


def cache(**kw):
    f = {"k": A, "v": A, "k_scale": A, "v_scale": A, "k_bounds": A, "pages": 8, "heads": 2, "page_tokens": 16, "d": 64, "code_type": 0}
    f.update(kw)
    return tq.Kv8(*f.values())


def append(c, **kw):
    f = {"table": A, "ldt": 4, "width": 4, "nseq": 2, "tokens": A, "starts": A, "n": 5, "K": A, "ldk": 128, "hk": 64, "V": A, "ldv": 128, "hv": 64,
         "dtype": 0}
    f.update(kw)
    return tq.lib().tq_kv8_append(ctypes.byref(c) if c else None, *f.values(), None)


def attend(c, **kw):
    f = {"table": A, "ldt": 4, "width": 4, "nseq": 2, "tokens": A, "starts": A, "n": 5, "max_queries": 3, "Q": A, "ldq": 512, "hq": 64, "g": 4, "dtype": 0,
         "scale": 1.0, "lists": None, "nlist": 0, "out": A, "ldo": 512, "ho": 64, "lse": A, "ws": None, "bytes": 0}
    f.update(kw)
    return tq.lib().tq_kv8_attend(ctypes.byref(c) if c else None, *f.values(), None)


def select(c, **kw):
    f = {"table": A, "ldt": 4, "width": 4, "nseq": 2, "tokens": A, "starts": A, "n": 5, "Q": A, "ldq": 512, "hq": 64, "g": 4, "dtype": 0, "first": 1,
         "last": 1, "k": 3, "lists": A, "ws": A, "bytes": 1 << 20}
    f.update(kw)
    return tq.lib().tq_kv8_select(ctypes.byref(c) if c else None, *f.values(), None)


@pytest.mark.parametrize("call", [append, attend, select])
def test_cache_and_batch(call):
    assert call(None) == INVALID
    assert call(cache(code_type=2)) == UNSUPPORTED
    for d in (0, 16, 48, 160, 256):
        assert call(cache(d=d)) == UNSUPPORTED
    for t in (0, 8, 48, 256):
        assert call(cache(page_tokens=t)) == UNSUPPORTED
    assert call(cache(heads=0)) == UNSUPPORTED and call(cache(heads=70000)) == UNSUPPORTED
    assert call(cache(pages=-1)) == INVALID and call(cache(k=None)) == INVALID and call(cache(v_scale=None)) == INVALID
    assert call(cache(v=A + 8)) == ALIGNMENT and call(cache(k_bounds=A + 4)) == ALIGNMENT
    assert b"aligned" in tq.lib().tq_last_error()
    c = cache()
    assert call(c, nseq=-1) == INVALID and call(c, n=-1) == INVALID and call(c, width=5) == INVALID
    assert call(c, tokens=None) == INVALID and call(c, table=None) == INVALID
    assert call(c, starts=None) == INVALID                      # 5 rows for 2 sequences
    assert call(c, n=1 << 31) == UNSUPPORTED and call(c, nseq=(1 << 20) + 1) == UNSUPPORTED
    assert call(c, dtype=2) == UNSUPPORTED
    assert call(c, n=0) == 0 and call(c, nseq=0, n=0) == 0      # nothing to do


def test_append():
    c = cache()
    assert append(c, K=None) == INVALID and append(c, V=None) == INVALID
    assert append(c, ldk=-1) == INVALID and append(c, hv=-64) == INVALID
    assert append(c, K=A + 2) == ALIGNMENT and append(c, V=A + 1, dtype=1) == ALIGNMENT


def test_attend():
    c = cache()
    assert attend(c, g=0) == UNSUPPORTED and attend(c, g=257) == UNSUPPORTED
    assert attend(c, max_queries=-1) == INVALID and attend(c, nlist=3) == INVALID and attend(c, lists=A, nlist=-1) == INVALID and attend(c, lists=A, nlist=0) == INVALID
    assert attend(c, starts=None, n=2, max_queries=0) == INVALID
    assert attend(c, Q=None) == INVALID and attend(c, out=None) == INVALID
    assert attend(c, ldo=-1) == INVALID
    assert attend(c, out=A + 2) == ALIGNMENT and attend(c, Q=A + 1, dtype=1) == ALIGNMENT and attend(c, lse=A + 2) == ALIGNMENT
    assert attend(c, ws=None) == WORKSPACE
    assert attend(c, max_queries=0) == 0


def test_select():
    c = cache()
    assert select(c, g=0) == UNSUPPORTED and select(c, g=300) == UNSUPPORTED
    assert select(c, k=0) == INVALID and select(c, first=2, last=2) == INVALID and select(c, first=-1) == INVALID
    assert select(c, Q=None) == INVALID and select(c, lists=None) == INVALID
    assert select(cache(k_bounds=None)) == INVALID and b"bounds" in tq.lib().tq_last_error()
    assert select(c, lists=A + 2) == ALIGNMENT and select(c, Q=A + 2) == ALIGNMENT and select(c, ws=A + 128) == ALIGNMENT
    need = tq.lib().tq_kv8_select_workspace_bytes(ctypes.byref(c), 5, 4)
    assert need == 5 * 2 * 4 * 4 and select(c, bytes=need - 1) == WORKSPACE and select(c, ws=None) == WORKSPACE


def test_pages():
    L = tq.lib()
    c = ctypes.byref(cache())
    need = L.tq_pages_workspace_bytes(8, 2)
    assert need > 0 and L.tq_pages_workspace_bytes(-1, 2) == 0
    extend = lambda refs=A, pages=8, table=A, ldt=4, width=4, rows=2, tokens=A, nxt=A, t=16, spare=A, ws=A, n=need: L.tq_pages_extend(
        refs, pages, table, ldt, width, rows, tokens, nxt, t, spare, ws, n, None)
    assert extend(refs=None) == INVALID and extend(pages=-1) == INVALID and extend(table=None) == INVALID and extend(ldt=3) == INVALID
    assert extend(tokens=None) == INVALID and extend(nxt=None) == INVALID and extend(spare=None) == INVALID
    assert extend(t=24) == UNSUPPORTED and extend(rows=(1 << 20) + 1) == UNSUPPORTED and extend(rows=1 << 20, width=1 << 12, ldt=1 << 12) == UNSUPPORTED
    assert extend(n=need - 1) == WORKSPACE and extend(ws=None) == WORKSPACE and extend(ws=A + 16) == ALIGNMENT
    assert extend(rows=0) == 0
    fork = lambda cc=c, refs=A, table=A, tokens=A, parents=A, children=A, count=2, spare=A, ws=A, n=need: L.tq_pages_fork(
        cc, refs, table, 4, 4, 2, tokens, parents, children, count, spare, ws, n, None)
    assert fork(cc=None) == INVALID and fork(refs=None) == INVALID and fork(table=None) == INVALID and fork(tokens=None) == INVALID
    assert fork(parents=None) == INVALID and fork(children=None) == INVALID and fork(count=-1) == INVALID and fork(spare=None) == INVALID
    assert fork(n=8) == WORKSPACE and fork(count=0) == 0
    assert L.tq_pages_free(None, 8, A, 4, 4, 2, A, A, 1, None) == INVALID
    assert L.tq_pages_free(A, 8, A, 4, 4, 2, A, None, 1, None) == INVALID and L.tq_pages_free(A, 8, A, 4, 4, 2, A, A, -1, None) == INVALID
    assert L.tq_pages_free(A, 8, A, 4, 4, 2, None, None, 0, None) == 0
    assert L.tq_pages_compact(c, A, A, 4, 4, 2, None, A, need, None) == INVALID and L.tq_pages_compact(c, A, A, 4, 4, 2, A, A, 16, None) == WORKSPACE
    assert L.tq_pages_copy(c, None, A, 1, None) == INVALID and L.tq_pages_copy(c, A, A, -1, None) == INVALID and L.tq_pages_copy(c, A, A, 0, None) == 0


def test_tensors_of_the_host_are_refused():
    k = torch.zeros((4, 2, 16, 32), dtype=torch.int8)
    s = torch.zeros((4, 2))
    with pytest.raises(ValueError):
        tq.Kv8Cache(k, k.clone(), s, s.clone())
    with pytest.raises(ValueError):
        tq.Kv8Cache(k.float(), k.float(), s, s.clone())
    with pytest.raises(ValueError):
        tq.tq_pages_free(torch.zeros(4, dtype=torch.int32), torch.zeros((1, 4), dtype=torch.int32), None, torch.zeros(1, dtype=torch.int32))


@pytest.mark.parametrize("call", [append, attend, select])
def test_tables_of_more_tokens_than_32_bits_count(call):
    for t in (16, 32, 64, 128):
        most = min(1 << 24, ((1 << 31) - 256) // t)
        for width in (most, most + 1):
            rc = call(cache(page_tokens=t), width=width, ldt=width, n=0)
            assert rc == (0 if width == most else UNSUPPORTED)
