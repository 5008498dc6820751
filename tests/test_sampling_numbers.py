"""Settings and counts of other types than Python's numbers: numpy's scalars are numbers like any, what is none is
refused as a value."""
import decimal

import numpy as np
import pytest

from test_sampling_binding import I32, T, calls, plan, probs, verify  # noqa: F401 (the fixture of that module)


@pytest.mark.parametrize("number", [np.float32(0.5), np.float64(0.5), np.float16(0.5), np.array(0.5), decimal.Decimal("0.5")])
@pytest.mark.parametrize("name", ["temperature", "top_p"])
def test_numbers(calls, name, number):  # noqa: F811
    m, _, seen = calls
    del seen[:]
    probs(m, **{name: number})
    assert len(seen) == 1


@pytest.mark.parametrize("number", [np.int64(3), np.int32(3), np.uint8(3), np.array(3), True, 1 << 100])
def test_whole_numbers(calls, number):  # noqa: F811
    m, _, seen = calls
    del seen[:]
    probs(m, top_k=number)
    probs(m, temperature=0 if number == 1 << 100 else number, top_p=1 if number == 1 << 100 else number)
    if number != 1 << 100:
        plan(m, rows=number, n_rows=number)
        assert seen[-1][3] == seen[-1][4] == int(number)
        verify(m, draft_start=T((3,), I32), max_drafts=number)
    assert len(seen) == (2 if number == 1 << 100 else 4)


@pytest.mark.parametrize("kw", [dict(temperature=np.float32(-1)), dict(temperature=np.float32("nan")), dict(temperature="1"),
                                dict(temperature=np.array([0.5, 0.5])), dict(temperature=[0.5]), dict(temperature=1j),
                                dict(temperature=None), dict(temperature=10 ** 400), dict(top_k=np.float32(3)),
                                dict(top_k=3.0), dict(top_k=np.int64(-1)), dict(top_k=np.array([1, 2])), dict(top_k="3"),
                                dict(top_k=-(1 << 100)), dict(top_p=np.float32(-0.5)), dict(top_p="x"), dict(top_p=np.ones(4))])
def test_what_is_no_number_is_refused(calls, kw):  # noqa: F811
    m, _, seen = calls
    del seen[:]
    with pytest.raises(ValueError):
        probs(m, **kw)
    assert not seen


@pytest.mark.parametrize("kw", [dict(rows=1.5), dict(rows="3"), dict(rows=np.int64(-1)), dict(rows=1 << 100), dict(n_rows=1.5),
                                dict(n_rows="3"), dict(n_rows=1 << 100)])
def test_counts_that_are_none_are_refused(calls, kw):  # noqa: F811
    m, _, seen = calls
    del seen[:]
    with pytest.raises(ValueError):
        plan(m, **kw)
    assert not seen


def test_max_drafts(calls):  # noqa: F811
    m, _, seen = calls
    del seen[:]
    for bad in ("2", 2.5, 1 << 100, np.int64(-1)):
        with pytest.raises(ValueError):
            verify(m, max_drafts=bad)
    assert not seen


@pytest.mark.gpu
def test_they_count_as_what_they_are():
    import torch
    from paper_2510_05421_gb300 import PagePool, token_probs
    x = torch.randn(3, 3001, generator=torch.Generator().manual_seed(0)).cuda()
    got = token_probs(x, np.float32(0.75), np.int64(50), np.array(0.875))
    assert torch.equal(got, token_probs(x, 0.75, 50, 0.875))
    assert torch.equal(token_probs(x, 1.0, 1 << 100), token_probs(x))
    pool = PagePool.create(np.int64(8), np.int64(2), np.int64(4), np.int64(16))
    plan = pool.plan(torch.tensor([3, 16], dtype=torch.int32).cuda(), np.int64(20), n_rows=np.int64(40))
    assert plan.row_start.tolist() == [0, 20, 40] and pool.held.tolist() == [2, 3] and pool.status() == []
