"""The paged cache's Python side without a GPU: the module builds and loads, and its checks refuse what the library
cannot take, on stand-ins for tensors and a library that only counts its calls."""
import ctypes
import os

import pytest
import torch

from paper_2510_05421_gb300 import build as build_mod
from paper_2510_05421_gb300.paged import PagedCacheC

A = 1 << 20


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
    if not os.path.exists(build_mod.PY_OUT):
        build_mod.build_py()
    loader = importlib.machinery.ExtensionFileLoader("_paged", build_mod.PY_OUT)
    m = importlib.util.module_from_spec(importlib.util.spec_from_loader("_paged", loader))
    loader.exec_module(m)
    seen = []
    vp, i, ll, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t
    types = ([vp, vp, i, vp, ll, vp, ll, vp, i, i, vp, ll, vp, ll, i, vp], [vp, vp, vp, i, vp, ll, vp, ll, vp, sz, vp],
             [vp, vp, i, vp, vp, vp])
    fns = [ctypes.CFUNCTYPE(i, *t)(lambda *a: (seen.append(a), 7)[1]) for t in types]
    m.init(*[ctypes.cast(f, vp).value for f in fns], torch.int32, torch.float32, torch.bfloat16)
    m_keep = (m, fns, seen)
    yield m_keep
    # the process's own module is the same object file: give it its library back
    from paper_2510_05421_gb300 import paged
    paged._calls = None
    paged._module()


C = PagedCacheC(8, 2, 16, 64, 0, A, A, A, A)
AT = (ctypes.addressof(C), 0, A)
I32, F32, BF = torch.int32, torch.float32, torch.bfloat16


def table(B=2, w=4, **kw):
    return T((B, w), kw.pop("dtype", I32), **kw)


def rows(n=4, h=2, D=64, dtype=BF, **kw):
    return T((n, h, D), dtype, **kw)


def attend(m, **kw):
    a = dict(table=table(), lens=T((2,), I32), q=rows(h=4), out=rows(h=4), scale=0.1, softcap=0.0, window=0, slopes=None,
             row_start=None, max_rows=None)
    a.update(kw)
    return m.attend(*AT, a["table"], a["lens"], a["q"], a["out"], a["scale"], a["softcap"], a["window"], a["slopes"],
                    a["row_start"], a["max_rows"], A, 4096, 0)


def append(m, **kw):
    a = dict(table=table(), lens=T((2,), I32), k=rows(), v=rows(), q=None, rotary=None, row_start=None, max_rows=None,
             q_out=None)
    a.update(kw)
    return m.append(*AT, a["table"], a["lens"], a["k"], a["v"], a["q"], a["rotary"], a["row_start"], a["max_rows"],
                    a["q_out"], 0)


def test_good_calls_reach_the_library(calls):
    m, _, seen = calls
    del seen[:]
    assert attend(m) == 7 and append(m) == 7 and m.read(*AT, table(), T((2,), I32), rows(), rows(), None, None, 0) == 7
    assert attend(m, row_start=T((3,), I32), max_rows=3, slopes=T((4,), F32), window=5, softcap=2.0) == 7
    assert append(m, q=rows(h=6), q_out=rows(h=6), rotary=T((9, 16, 2), F32)) == 7
    wide = (1000, 64, 1)                                    # rows of a projection's output lie apart
    assert append(m, k=rows(stride=wide), v=rows(stride=wide)) == 7
    assert seen[-1][4] == 1000 and len(seen) == 6
    assert attend(m, q=rows(n=0, h=4), out=rows(n=0, h=4)) == 7


BAD = [dict(q=rows(h=4, dtype=torch.float16)), dict(q=rows(h=3), out=rows(h=3)), dict(q=rows(h=4, D=32)),
       dict(q=rows(h=4, device=-1)), dict(q=T((4, 64), BF)), dict(q=rows(h=4, stride=(64, 256, 1))),
       dict(q=rows(h=4, ptr=A + 8)), dict(out=rows(n=3, h=4)), dict(out=rows(h=4, dtype=F32)),
       dict(out=rows(h=4, stride=(257, 64, 1))), dict(scale=0.0), dict(scale=float("nan")), dict(softcap=-1.0),
       dict(softcap=float("inf")), dict(window=-1), dict(window=1 << 31), dict(slopes=T((3,), F32)),
       dict(slopes=T((4,), BF)), dict(table=table(dtype=torch.int64)), dict(table=T((8,), I32)),
       dict(table=table(device=1)), dict(table=table(stride=(8, 1))), dict(lens=T((3,), I32)),
       dict(lens=T((2,), torch.int64)), dict(table=table(3), lens=T((3,), I32)), dict(row_start=T((2,), I32)),
       dict(row_start=T((3,), torch.int64)), dict(row_start=T((3,), I32), max_rows=-1), dict(table=table(w=(1 << 26) + 1)),
       dict(table=table(2000), lens=T((2000,), I32), row_start=T((2001,), I32))]


@pytest.mark.parametrize("kw", BAD)
def test_attend_refuses(calls, kw):
    m, _, seen = calls
    del seen[:]
    with pytest.raises(ValueError):
        attend(m, **kw)
    assert not seen


@pytest.mark.parametrize("kw", [dict(k=rows(h=3)), dict(v=rows(dtype=F32)), dict(v=rows(n=3)), dict(k=rows(ptr=A + 4)),
                                dict(k=rows(stride=(132, 64, 1))), dict(q=rows(h=4)), dict(q_out=rows(h=4)),
                                dict(q=rows(n=2, h=4), q_out=rows(n=2, h=4)), dict(rotary=T((9, 16, 2), BF)),
                                dict(rotary=T((9, 12, 2), F32)), dict(rotary=T((9, 40, 2), F32)),
                                dict(rotary=T((0, 16, 2), F32)), dict(rotary=T((9, 16), F32))])
def test_append_refuses(calls, kw):
    m, _, seen = calls
    del seen[:]
    with pytest.raises(ValueError):
        append(m, **kw)
    assert not seen


def test_what_is_not_a_tensor_is_an_error(calls):
    m = calls[0]
    for kw in (dict(q=None), dict(table=5), dict(lens="x")):
        with pytest.raises((AttributeError, ValueError)):
            attend(m, **kw)
    with pytest.raises(TypeError):
        m.attend(1, 2)
