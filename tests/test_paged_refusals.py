"""The paged cache's C entry points refuse what they cannot take, by status code and before any device work
(no GPU here: the pointers are never followed)."""
import ctypes

import pytest

from paper_2510_05421_gb300 import build as build_mod
from paper_2510_05421_gb300 import dvi as D
from paper_2510_05421_gb300.paged import PagedBatchC, PagedCacheC, PagedOptionsC

A = 1 << 20     # an aligned address that nobody reads


@pytest.fixture(scope="module")
def L():
    import os
    if not os.path.exists(D.LIB_PATH):
        build_mod.build()
    return D.lib()


def cache(**kw):
    f = dict(n_pages=8, n_kv_heads=2, page_tokens=16, head_dim=64, format=0, k=A, v=A, k_scale=A, v_scale=A)
    f.update(kw)
    return PagedCacheC(*[f[n] for n, _ in PagedCacheC._fields_])


def batch(**kw):
    f = dict(n_seqs=2, max_pages=4, n_rows=4, max_rows=2, table=A, lens=A, row_start=None, status=None)
    f.update(kw)
    return PagedBatchC(*[f[n] for n, _ in PagedBatchC._fields_])


def options(**kw):
    f = dict(n_heads=4, scale=0.1, softcap=0.0, window=0, slopes=None)
    f.update(kw)
    return PagedOptionsC(*[f[n] for n, _ in PagedOptionsC._fields_])


def calls(L, c, b, dtype=1):
    r = ctypes.byref
    yield L.dvi_paged_append(r(c), r(b), dtype, A, 128, A, 128, None, 0, 0, None, 0, None, 0, 0, None)
    yield L.dvi_paged_attend(r(c), r(b), r(options()), dtype, A, 256, A, 256, A, 1 << 40, None)
    yield L.dvi_paged_read(r(c), r(b), dtype, A, A, None)


BAD_CACHE = [dict(n_pages=0), dict(n_kv_heads=0), dict(n_kv_heads=1025), dict(page_tokens=8), dict(page_tokens=48),
             dict(head_dim=96), dict(format=2), dict(k=None), dict(v=A + 8), dict(k_scale=None), dict(v_scale=A + 4)]
BAD_BATCH = [dict(n_seqs=0), dict(max_pages=0), dict(n_rows=-1), dict(max_rows=-1), dict(table=None), dict(lens=None),
             dict(n_rows=5), dict(max_rows=1)]
TOO_LARGE = [dict(n_seqs=1025, row_start=A), dict(max_pages=(1 << 26) + 1), dict(n_rows=(1 << 30) + 2, max_rows=1 << 30)]


@pytest.mark.parametrize("kw", BAD_CACHE)
def test_bad_cache(L, kw):
    assert list(calls(L, cache(**kw), batch())) == [-1, -1, -1]


@pytest.mark.parametrize("kw", BAD_BATCH)
def test_bad_batch(L, kw):
    assert list(calls(L, cache(), batch(**kw))) == [-1, -1, -1]


@pytest.mark.parametrize("kw", TOO_LARGE)
def test_too_large(L, kw):
    assert list(calls(L, cache(), batch(**kw))) == [-2, -2, -2]


def test_bad_type_and_null(L):
    assert list(calls(L, cache(), batch(), dtype=2)) == [-1, -1, -1]
    r = ctypes.byref
    assert L.dvi_paged_append(None, r(batch()), 1, A, 128, A, 128, None, 0, 0, None, 0, None, 0, 0, None) == -1
    assert L.dvi_paged_attend(r(cache()), None, r(options()), 1, A, 256, A, 256, A, 1 << 40, None) == -1
    assert L.dvi_paged_attend(r(cache()), r(batch()), None, 1, A, 256, A, 256, A, 1 << 40, None) == -1
    assert L.dvi_paged_read(r(cache()), r(batch()), 1, None, A, None) == -1


@pytest.mark.parametrize("args", [
    (None, 128, A, 128, None, 0, 0, None, 0, None, 0, 0),      # no k
    (A, 127, A, 128, None, 0, 0, None, 0, None, 0, 0),         # rows closer than their heads
    (A, 132, A, 128, None, 0, 0, None, 0, None, 0, 0),         # rows off 16 bytes
    (A, 128, A + 2, 128, None, 0, 0, None, 0, None, 0, 0),     # v off 16 bytes
    (A, 128, A, 128, A, 24, 9, None, 0, None, 0, 0),           # rot_dim
    (A, 128, A, 128, A, 80, 9, None, 0, None, 0, 0),
    (A, 128, A, 128, A, 64, 0, None, 0, None, 0, 0),           # an empty table
    (A, 128, A, 128, None, 0, 0, A, 256, None, 256, 4),        # q without q_out
    (A, 128, A, 128, None, 0, 0, A, 255, A, 256, 4),
    (A, 128, A, 128, None, 0, 0, A, 256, A, 256, 0),
])
def test_bad_append(L, args):
    r = ctypes.byref
    assert L.dvi_paged_append(r(cache()), r(batch()), 1, *args, None) == -1


@pytest.mark.parametrize("kw", [dict(n_heads=0), dict(n_heads=3), dict(scale=0.0), dict(scale=float("nan")),
                                dict(scale=float("inf")), dict(softcap=-1.0), dict(softcap=float("nan")),
                                dict(window=-1)])
def test_bad_options(L, kw):
    r = ctypes.byref
    assert L.dvi_paged_attend(r(cache()), r(batch()), r(options(**kw)), 1, A, 512, A, 512, A, 1 << 40, None) == -1


@pytest.mark.parametrize("args", [(None, 256, A, 256, A), (A, 256, None, 256, A), (A, 255, A, 256, A),
                                  (A, 256, A, 260, A), (A + 4, 256, A, 256, A), (A, 256, A, 256, None),
                                  (A, 256, A, 256, A + 128)])
def test_bad_attend(L, args):
    r = ctypes.byref
    q, ldq, o, ldo, ws = args
    assert L.dvi_paged_attend(r(cache()), r(batch()), r(options()), 1, q, ldq, o, ldo, ws, 1 << 40, None) == -1


def test_workspace_of_unknown_head_dim(L):
    assert L.dvi_paged_workspace_bytes(96) == 0
