"""Caps so far below the scale that scale / softcap leaves f32 (or the cap itself does) are refused, by the C entry and by
the binding: a cap that became 0 on the way would be none, and 0 times an infinity no score."""
import ctypes

import pytest

from test_paged_binding import attend, calls  # noqa: F401
from test_paged_refusals import A, L, batch, cache, options  # noqa: F401

BAD = [dict(softcap=1e-39), dict(softcap=1e-32, scale=0.1), dict(softcap=1e-8, scale=1e24)]
GOOD = [dict(softcap=1e-28), dict(softcap=1e-8, scale=1e20), dict(softcap=0.0), dict(softcap=9e29)]


def call(lib, kw):
    """The status without a workspace large enough, which ends a call whose options are good before any launch."""
    r = ctypes.byref
    return lib.dvi_paged_attend(r(cache()), r(batch()), r(options(**kw)), 1, A, 256, A, 256, A, 0, None)


@pytest.mark.parametrize("kw", BAD)
def test_c_entry_refuses(L, kw):  # noqa: F811
    assert call(L, kw) == -1


@pytest.mark.parametrize("kw", GOOD)
def test_c_entry_looks_further(L, kw):  # noqa: F811
    assert call(L, kw) in (-2, -4)         # DVI_ERR_CAPACITY; DVI_ERR_CUDA without a GPU


@pytest.mark.parametrize("kw", BAD + [dict(softcap=1e-46), dict(scale=1e-50)])
def test_binding_refuses(calls, kw):  # noqa: F811
    m, _, seen = calls
    del seen[:]
    with pytest.raises(ValueError):
        attend(m, **kw)
    assert not seen


@pytest.mark.parametrize("kw", GOOD)
def test_binding_passes_on(calls, kw):  # noqa: F811
    assert attend(calls[0], **kw) == 7
