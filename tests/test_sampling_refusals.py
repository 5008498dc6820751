"""The C entry points of page plans and sampling refuse what they cannot take, by status code and before any device
work (no GPU here: the pointers are never followed)."""
import ctypes

import pytest

from paper_2510_05421_gb300 import build as build_mod
from paper_2510_05421_gb300 import dvi as D
from paper_2510_05421_gb300.pages import PagePoolC

A = 1 << 20     # an aligned address that nobody reads
NAN = float("nan")


class Sampling(ctypes.Structure):
    _fields_ = [("temperature", ctypes.c_void_p), ("top_k", ctypes.c_void_p), ("top_p", ctypes.c_void_p),
                ("temperature_all", ctypes.c_float), ("top_k_all", ctypes.c_int), ("top_p_all", ctypes.c_float)]


class Drafts(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("n_seqs", "vocab", "n_drafts", "max_drafts", "bonus")] + [
        (n, ctypes.c_void_p) for n in ("draft_start", "draft_ids", "u_accept", "u_token", "status")]


@pytest.fixture(scope="module")
def L():
    import os
    if not os.path.exists(D.LIB_PATH):
        build_mod.build()
    return D.lib()


def probs(L, **kw):
    a = dict(dtype=0, x=A, ld=100, n=4, vocab=100, out=A, ld_out=100, status=None, temperature=None, top_k=None, top_p=None,
             temperature_all=1.0, top_k_all=0, top_p_all=1.0)
    a.update(kw)
    s = Sampling(*[a[n] for n, _ in Sampling._fields_])
    return L.dvi_token_probs(a["dtype"], a["x"], a["ld"], a["n"], a["vocab"], ctypes.byref(s), a["out"], a["ld_out"],
                             a["status"], None)


@pytest.mark.parametrize("kw", [dict(dtype=2), dict(x=None), dict(x=A + 2), dict(dtype=1, x=A + 1), dict(out=None),
                                dict(out=A + 2), dict(ld=99), dict(ld_out=99), dict(n=-1), dict(vocab=0), dict(status=A + 2),
                                dict(temperature=A + 1), dict(top_k=A + 2), dict(top_p=A + 3), dict(temperature_all=-1.0),
                                dict(temperature_all=NAN), dict(top_k_all=-1), dict(top_p_all=-0.5), dict(top_p_all=NAN)])
def test_token_probs(L, kw):
    assert probs(L, **kw) == -1


def test_token_probs_sizes(L):
    assert probs(L, vocab=(1 << 18) + 1, ld=1 << 20, ld_out=1 << 20) == -2
    assert probs(L, n=(1 << 30) + 1) == -2
    assert probs(L, n=0) == 0 and probs(L, n=0, x=None, out=None) == 0
    assert L.dvi_token_probs(0, A, 100, 4, 100, None, A, 100, None, None) == -1


def verify(L, **kw):
    a = dict(n_seqs=2, vocab=50, n_drafts=4, max_drafts=2, bonus=1, draft_start=None, draft_ids=A, u_accept=A, u_token=A,
             status=None, p=A, ld_p=50, q=A, ld_q=50, out=A, nc=A, na=A)
    a.update(kw)
    b = Drafts(*[a[n] for n, _ in Drafts._fields_])
    return L.dvi_verify_drafts(ctypes.byref(b), a["p"], a["ld_p"], a["q"], a["ld_q"], a["out"], a["nc"], a["na"], None)


@pytest.mark.parametrize("kw", [dict(n_seqs=-1), dict(vocab=0), dict(n_drafts=-1), dict(max_drafts=-1), dict(bonus=2),
                                dict(n_drafts=5), dict(max_drafts=1), dict(n_seqs=0), dict(draft_ids=None),
                                dict(u_accept=None), dict(u_token=None), dict(p=None), dict(ld_p=49), dict(ld_q=49),
                                dict(q=A + 2), dict(p=A + 1), dict(out=None), dict(out=A + 2), dict(nc=None), dict(na=None),
                                dict(na=A + 2), dict(status=A + 1), dict(draft_start=A + 2), dict(draft_ids=A + 2)])
def test_verify_drafts(L, kw):
    assert verify(L, **kw) == -1


@pytest.mark.parametrize("kw", [dict(n_seqs=65537, n_drafts=0), dict(vocab=(1 << 18) + 1, ld_p=1 << 20, ld_q=1 << 20),
                                dict(n_drafts=(1 << 30) + 2, max_drafts=1 << 20), dict(max_drafts=(1 << 20) + 1)])
def test_verify_drafts_sizes(L, kw):
    assert verify(L, **kw) == -2


def test_verify_nothing(L):
    assert verify(L, n_seqs=0, n_drafts=0) == 0
    assert L.dvi_verify_drafts(None, A, 50, A, 50, A, A, A, None) == -1


def plan(L, lens=A, rows=A, each=0, n_rows=8, start=A, slots=A, positions=A, **kw):
    f = dict(n_pages=8, page_tokens=16, n_seqs=2, max_pages=4, stack=A, n_free=A, table=A, held=A, status=None)
    f.update(kw)
    c = PagePoolC(*[f[n] for n, _ in PagePoolC._fields_])
    return L.dvi_paged_plan(ctypes.byref(c), lens, rows, each, n_rows, start, slots, positions, None)


@pytest.mark.parametrize("kw", [dict(n_pages=0), dict(page_tokens=8), dict(page_tokens=48), dict(n_seqs=0), dict(max_pages=0),
                                dict(stack=None), dict(n_free=None), dict(table=None), dict(held=None), dict(lens=None),
                                dict(stack=A + 2), dict(status=A + 1), dict(rows=A + 2), dict(slots=A + 4), dict(start=A + 1),
                                dict(positions=A + 2), dict(n_rows=-1), dict(each=-1)])
def test_paged_plan(L, kw):
    assert plan(L, **kw) == -1


@pytest.mark.parametrize("kw", [dict(n_seqs=1025), dict(max_pages=(1 << 26) + 1), dict(n_rows=(1 << 30) + 1),
                                dict(each=(1 << 30) + 1)])
def test_paged_plan_sizes(L, kw):
    assert plan(L, **kw) == -2


def test_paged_plan_of_nothing(L):
    assert L.dvi_paged_plan(None, A, A, 0, 8, A, A, A, None) == -1


@pytest.mark.parametrize("kw", [dict(out=A + 4), dict(out=A - 4), dict(out=A + 400), dict(out=A + 1600 - 4), dict(ld=128),
                                dict(ld_out=128, out=A + 256), dict(dtype=1), dict(dtype=1, ld=200, out=A + 4),
                                dict(ld=210, ld_out=210, out=A + 396), dict(ld=210, ld_out=210, out=A + 210 * 4 - 4),
                                dict(n=1, out=A + 4), dict(n=1, dtype=1)])
def test_probabilities_over_their_own_logits(L, kw):
    """Rows that share memory and are not the same: 100 numbers of 4 (logits in bf16: 2) bytes a row."""
    assert probs(L, **kw) == -1
