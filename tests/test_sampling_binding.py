"""The Python side of page plans and sampling without a GPU: its checks refuse what the library cannot take, on
stand-ins for tensors and a library that only counts its calls."""
import ctypes
import os

import pytest
import torch

from paper_2510_05421_gb300 import build as build_mod
from paper_2510_05421_gb300.pages import PagePoolC

A = 1 << 20
I32, I64, F32, BF = torch.int32, torch.int64, torch.float32, torch.bfloat16
NAN = float("nan")


class T:
    """What the checks ask of a tensor."""

    def __init__(self, shape, dtype, stride=None, device=0, ptr=A):
        step, run = [], 1
        for n in reversed(shape):
            step.insert(0, run)
            run *= n
        self.shape, self.dtype = torch.Size(shape), dtype
        self._s, self._d, self._p = tuple(stride or step), device, ptr

    def stride(self):
        return self._s

    def get_device(self):
        return self._d

    def data_ptr(self):
        return self._p


@pytest.fixture(scope="module")
def calls():
    """A copy of the module whose library only records its last call's arguments."""
    import importlib.machinery
    import importlib.util
    if not os.path.exists(build_mod.PY_SAMPLING_OUT):
        build_mod.build_py()
    loader = importlib.machinery.ExtensionFileLoader("_sampling", build_mod.PY_SAMPLING_OUT)
    m = importlib.util.module_from_spec(importlib.util.spec_from_loader("_sampling", loader))
    loader.exec_module(m)
    seen = []
    vp, i, ll = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64
    types = ([i, vp, ll, i, i, vp, vp, ll, vp, vp], [vp, vp, ll, vp, ll, vp, vp, vp, vp], [vp, vp, vp, i, i, vp, vp, vp, vp])
    answer = [0]
    fns = [ctypes.CFUNCTYPE(i, *t)(lambda *a: (seen.append(a), answer[0])[1]) for t in types]
    m.init(*[ctypes.cast(f, vp).value for f in fns], I32, I64, F32, BF, lambda n, step, dt: T(n, dt, step, ptr=B), Error)
    yield m, answer, seen
    # the process's own module is the same object file: give it its library back
    from paper_2510_05421_gb300 import sampling
    sampling._calls = None
    sampling._module()


class Error(RuntimeError):
    pass


B = 1 << 21     # of what a call makes


def probs(m, **kw):
    a = dict(logits=T((4, 100), F32), temperature=1.0, top_k=0, top_p=1.0, out=None, status=None)
    a.update(kw)
    return m.probs(*a.values(), 0)


def verify(m, **kw):
    a = dict(target=T((6, 50), F32), draft_ids=T((4,), I32), u_accept=T((4,), F32), u_token=T((2,), F32),
             draft=T((4, 50), F32), draft_start=None, max_drafts=2, bonus=True, status=None)
    a.update(kw)
    return m.verify(*a.values(), 0)


POOL = PagePoolC(8, 16, 2, 4, A, A, A, A, A)


def plan(m, **kw):
    a = dict(lens=T((2,), I32), rows=T((2,), I32), n_rows=8, starts=True)
    a.update(kw)
    return m.plan(ctypes.addressof(POOL), 0, *a.values(), 0)


def shapes(got):
    return [None if t is None else (tuple(t.shape), t.stride(), t.dtype) for t in got]


def test_good_calls_reach_the_library(calls):
    m, _, seen = calls
    del seen[:]
    assert shapes([probs(m), probs(m, logits=T((4, 100), BF), status=T((1,), I32))]) == [((4, 100), (100, 1), F32)] * 2
    assert seen[-1][6] == B and seen[-1][7] == 100
    probs(m, temperature=T((4,), F32), top_k=T((4,), I32), top_p=T((4,), F32))
    probs(m, temperature=0, top_k=1 << 40, top_p=7)
    out = T((4, 100), F32, stride=(101, 1))
    assert probs(m, logits=T((4, 100), F32, stride=(128, 1)), out=out) is out
    assert seen[-1][2] == 128 and seen[-1][6] == A and seen[-1][7] == 101
    probs(m, logits=T((0, 100), F32))
    one = ((2,), (1,), I32)
    assert shapes(verify(m)) == [((2, 3), (3, 1), I32), one, one]
    assert shapes(verify(m, draft=None, status=T((1,), I32))) == shapes(verify(m, max_drafts=None)) == shapes(verify(m))
    assert shapes(verify(m, bonus=False, target=T((4, 50), F32)))[0] == ((2, 2), (2, 1), I32)
    assert shapes(verify(m, draft_start=T((3,), I32), max_drafts=5))[0] == ((2, 6), (6, 1), I32)
    assert shapes(verify(m, draft_ids=T((0,), I32), u_accept=T((0,), F32), draft=None, target=T((2, 50), F32),
                         max_drafts=0))[0] == ((2, 1), (1, 1), I32)
    assert shapes(plan(m)) == shapes(plan(m, rows=3)) == [((3,), (1,), I32), ((8,), (1,), I64), ((8,), (1,), I32)]
    assert shapes(plan(m, n_rows=None)) == [((3,), (1,), I32), None, None]
    assert seen[-1][5] == B and seen[-1][6] is None
    assert plan(m, n_rows=None, starts=False) == (None, None, None)
    assert len(seen) == 17


def test_the_librarys_errors_are_raised(calls):
    m, answer, _ = calls
    for rc, name in ((-2, "DVI_ERR_CAPACITY"), (-4, "DVI_ERR_CUDA"), (9, "9")):
        answer[0] = rc
        try:
            for call in (probs, verify, plan):
                with pytest.raises(Error, match=name):
                    call(m)
        finally:
            answer[0] = 0


@pytest.mark.parametrize("kw", [dict(logits=T((4, 100), torch.float16)), dict(logits=T((400,), F32)),
                                dict(logits=T((4, 100), F32, stride=(1, 4))), dict(logits=T((4, 100), F32, stride=(99, 1))),
                                dict(logits=T((4, 100), F32, device=-1)), dict(logits=T((4, 0), F32)),
                                dict(logits=T((1, 262145), F32)), dict(temperature=-1.0),
                                dict(temperature=NAN), dict(temperature=T((3,), F32)), dict(temperature=T((4,), BF)),
                                dict(temperature=T((4,), F32, stride=(2,))), dict(temperature=T((4,), F32, device=1)),
                                dict(top_k=-1), dict(top_k=T((4,), I64)), dict(top_p=-1.0), dict(top_p=NAN),
                                dict(top_p=T((4, 1), F32)), dict(out=T((4, 100), BF)), dict(out=T((4, 99), F32)),
                                dict(out=T((4, 100), F32, device=1)), dict(out=T((4, 100), F32, stride=(50, 1))),
                                dict(status=T((2,), I32)), dict(status=T((1,), F32))])
def test_probs_refuses(calls, kw):
    m, _, seen = calls
    del seen[:]
    with pytest.raises(ValueError):
        probs(m, **kw)
    assert not seen


@pytest.mark.parametrize("kw", [dict(target=T((5, 50), F32)), dict(target=T((6, 50), BF)), dict(target=T((6, 50), F32, device=-1)),
                                dict(target=T((6, 50), F32, stride=(1, 6))), dict(draft_ids=T((4,), I64)),
                                dict(draft_ids=T((3,), I32)), dict(draft_ids=T((4,), I32, device=1)),
                                dict(u_accept=T((5,), F32)), dict(u_accept=T((4,), BF)), dict(u_token=T((3,), F32)),
                                dict(u_token=T((2,), I32)), dict(draft=T((4, 49), F32)), dict(draft=T((6, 50), F32)),
                                dict(draft=T((4, 50), BF)), dict(draft_start=T((2,), I32)), dict(draft_start=T((3,), I64)),
                                dict(max_drafts=1), dict(max_drafts=-1), dict(bonus=False),
                                dict(u_token=T((0,), F32)), dict(status=T((1,), I64)),
                                dict(draft_start=T((3,), I32), max_drafts=(1 << 20) + 1)])
def test_verify_refuses(calls, kw):
    m, _, seen = calls
    del seen[:]
    with pytest.raises(ValueError):
        verify(m, **kw)
    assert not seen


@pytest.mark.parametrize("kw", [dict(lens=T((3,), I32)), dict(lens=T((2,), I64)), dict(lens=T((2,), I32, device=1)),
                                dict(rows=T((3,), I32)), dict(rows=T((2,), F32)), dict(rows=-1), dict(rows=(1 << 30) + 1),
                                dict(n_rows=-1), dict(n_rows=(1 << 30) + 1)])
def test_plan_refuses(calls, kw):
    m, _, seen = calls
    del seen[:]
    with pytest.raises(ValueError):
        plan(m, **kw)
    assert not seen


def test_what_is_not_a_tensor_is_an_error(calls):
    m = calls[0]
    for call in (lambda: probs(m, logits=None), lambda: probs(m, top_k="x"), lambda: probs(m, top_k=1.5),
                 lambda: verify(m, draft_ids=[1, 2, 3, 4]), lambda: plan(m, lens=None)):
        with pytest.raises((AttributeError, ValueError)):
            call()
    with pytest.raises(TypeError):
        m.probs(1, 2)


def test_calls_on_cpu_tensors_are_refused():
    from paper_2510_05421_gb300 import PagePool, token_probs, verify_drafts
    x = torch.zeros(2, 10)
    with pytest.raises(ValueError):
        token_probs(x)
    with pytest.raises(ValueError):
        token_probs([1.0])
    with pytest.raises(ValueError):
        verify_drafts(x, torch.zeros(0, dtype=I32), x[0, :0], x[:, 0])
    i = lambda *s: torch.zeros(s, dtype=I32)
    with pytest.raises(ValueError):
        PagePool(i(8), i(1), i(2, 4), i(2), 16)
