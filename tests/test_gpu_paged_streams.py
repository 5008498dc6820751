"""Calls with a stream of their own beside work on the current one: memory that either stream still uses is not handed
out under it, and the call sees what the current stream was given before."""
import numpy as np
import pytest
import torch

from test_gpu_paged import host, ints, make_cache

pytestmark = pytest.mark.gpu
LONG = int(4e8)        # cycles: far longer than everything enqueued meanwhile
ROWS, HQ, D = 4000, 8, 64


def setup(fmt="int8"):
    cache = make_cache(fmt, 80, 2, 64, D, 1)
    q = torch.randn(ROWS, HQ, D, device="cuda").bfloat16()
    kv = torch.randn(ROWS, 2, D, device="cuda").bfloat16()
    return cache, ints(np.arange(80)[None]), ints([900]), q, kv


def calls(cache, table, lens, q, kv, stream):
    """Each call that makes tensors of its own, as (name, tensors)."""
    yield "append", lambda: (cache.append(table, lens, kv, kv, q=q, stream=stream),)
    yield "attend", lambda: (cache.attend(table, lens, q, stream=stream),)
    yield "read", lambda: cache.read(table, lens, ROWS, stream=stream)


@pytest.mark.parametrize("which", ["append", "attend", "read"])
def test_outputs_wait_for_the_current_streams_use_of_their_memory(which):
    """The output's memory was just given back by a tensor that pending work still reads."""
    cache, table, lens, q, kv = setup()
    side = torch.cuda.Stream()
    want = dict(calls(cache, table, lens, q, kv, None))[which]()
    got_shape = want[0].shape
    for _ in range(3):
        torch.cuda.synchronize()
        torch.cuda.empty_cache()
        old = [torch.ones(got_shape, dtype=torch.bfloat16, device="cuda") for _ in want]
        torch.cuda._sleep(LONG)
        kept = [x.clone() for x in old]
        del old
        got = dict(calls(cache, table, lens, q, kv, side))[which]()
        torch.cuda.synchronize()
        assert all((x == 1).all() for x in kept)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("which", ["append", "attend", "read"])
def test_dropped_outputs_are_not_handed_out_while_they_are_written(which):
    cache, table, lens, q, kv = setup()
    side = torch.cuda.Stream()
    shape = dict(calls(cache, table, lens, q, kv, None))[which]()[0].shape
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(LONG)
    dict(calls(cache, table, lens, q, kv, side))[which]()
    fresh = [torch.zeros(shape, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    assert all((x == 0).all() for x in fresh)


@pytest.mark.parametrize("which", ["append", "attend", "read"])
def test_dropped_inputs_are_not_handed_out_while_they_are_read(which):
    cache, table, lens, q, kv = setup()
    side = torch.cuda.Stream()
    want = dict(calls(cache, table, lens, q, kv, None))[which]()
    codes = host(cache)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(LONG)
    got = dict(calls(cache, table.clone(), lens.clone(), q.clone(), kv.clone(), side))[which]()
    fresh = [torch.full_like(x, 1) for x in (table, lens, q, kv, kv) for _ in range(2)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert all((host(cache)[x] == codes[x]).all() for x in ("k", "v", "k_scale", "v_scale"))
    assert len(fresh) == 10


def test_inputs_made_on_the_current_stream():
    """What is written there before the call is seen by it."""
    cache, table, lens, q, kv = setup()
    want = cache.attend(table, lens, q)
    side = torch.cuda.Stream()
    late = torch.zeros_like(q)
    torch.cuda.synchronize()
    torch.cuda._sleep(LONG)
    late.copy_(q)
    got = cache.attend(table, lens, late, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)


def test_the_current_stream_by_name_and_a_callers_out():
    cache, table, lens, q, _ = setup("e4m3")
    want = cache.attend(table, lens, q)
    assert torch.equal(cache.attend(table, lens, q, stream=torch.cuda.current_stream()), want)
    out, side = torch.zeros_like(q), torch.cuda.Stream()
    got = cache.attend(table, lens, q, out=out, stream=side)
    side.synchronize()
    assert got.data_ptr() == out.data_ptr() and torch.equal(out, want)


def test_a_stream_of_its_own_inside_a_capture():
    """The named stream joins the capture and is joined again."""
    cache, table, lens, q, _ = setup()
    want = cache.attend(table, lens, q)
    cache.attend(table, lens, q, stream=torch.cuda.Stream())
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = cache.attend(table, lens, q, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        out = out * 1
    out.zero_()
    graph.replay()
    assert torch.equal(out, want)


def test_a_captured_stream_from_outside_the_capture():
    cache, table, lens, q, _ = setup()
    want = cache.attend(table, lens, q)
    side, other, out = torch.cuda.Stream(), torch.cuda.Stream(), torch.zeros_like(q)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        with torch.cuda.stream(other):
            cache.attend(table, lens, q, out=out, stream=side)
    graph.replay()
    assert torch.equal(out, want)


def test_a_dropped_cache_is_not_handed_out_while_it_is_read():
    cache, table, lens, q, _ = setup()
    want = cache.attend(table, lens, q)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    shapes = [(x.shape, x.dtype) for x in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    with torch.cuda.stream(side):
        torch.cuda._sleep(LONG)
    got = cache.attend(table, lens, q, stream=side)
    del cache
    fresh = [torch.ones(s, dtype=t, device="cuda") for s, t in shapes for _ in range(2)]
    torch.cuda.synchronize()
    assert torch.equal(got, want) and len(fresh) == 8


def test_a_stream_of_another_device_is_refused():
    import types
    cache, table, lens, q, kv = setup()
    other = types.SimpleNamespace(device=torch.device("cuda", 7), cuda_stream=0)
    for name, call in calls(cache, table, lens, q, kv, other):
        with pytest.raises(ValueError):
            call()


def test_status_waits_for_every_stream():
    """Flags of a call still in flight on another stream are reported by the look, and only by that one."""
    cache, table, lens, _, kv = setup()
    bad = kv.clone()
    bad[5, 1, 3] = float("nan")
    side = torch.cuda.Stream()
    for _ in range(3):
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(LONG)
            cache.append(table, lens, bad, kv)
        assert cache.status() == ["NONFINITE"]
        assert cache.status() == []
        with torch.cuda.stream(side):
            cache.append(table, lens, bad, kv)
        assert cache.status() == ["NONFINITE"]
