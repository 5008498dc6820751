"""attend's workspace: captured calls have one of their own, cleared once a graph and only where it must be, replays run
beside other calls of the stream they were captured on, and caches share what a stream's calls use one after another."""
import ctypes
import gc

import numpy as np
import pytest
import torch

from paper_2510_05421_gb300 import lib
from test_gpu_paged import ints, make_cache

pytestmark = pytest.mark.gpu


def split_case(seed, D=64, ctx=12000):
    """A call whose groups are cut over many teams and joined through the workspace."""
    P = 64
    pages = -(-(ctx + 4) // P)
    cache = make_cache("int8", pages, 2, P, D, seed)
    q = torch.randn(4, 8, D, device="cuda").bfloat16()
    return cache, ints(np.arange(pages)[None]), ints([ctx]), q


def busy(graphs, streams, eager, want, times=40):
    """Replays on their streams and eager calls on the current one, all in flight together; every result looked at."""
    for _ in range(times):
        for (g, out), s in zip(graphs, streams):
            with torch.cuda.stream(s):
                out.zero_()
                g.replay()
        got = [eager() for _ in range(4)] if eager else []
        torch.cuda.synchronize()
        assert all(torch.equal(out, want) for _, out in graphs) and all(torch.equal(x, want) for x in got)


def capture(case, stream):
    cache, table, lens, q = case
    graph, out = torch.cuda.CUDAGraph(), torch.zeros_like(q)
    with torch.cuda.graph(graph, stream=stream):
        cache.attend(table, lens, q, out=out)
    return graph, out


def test_replays_beside_calls_on_the_stream_they_were_captured_on():
    case = split_case(1)
    cache, table, lens, q = case
    home, away = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(home):
        want = cache.attend(table, lens, q)
    torch.cuda.synchronize()
    graph = capture(case, home)
    with torch.cuda.stream(home):
        busy([graph], [away], lambda: cache.attend(table, lens, q), want)


def test_two_graphs_of_one_stream_replayed_on_two():
    case = split_case(2)
    cache, table, lens, q = case
    home, away = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(home):
        want = cache.attend(table, lens, q)
    torch.cuda.synchronize()
    graphs = [capture(case, home) for _ in range(2)]
    busy(graphs, [home, away], lambda: cache.attend(table, lens, q), want)


def test_a_graph_outlives_the_next_capture_and_its_cache_object():
    """What a later capture on the stream, and the end of the PagedCache, give back is not the graph's."""
    case = split_case(4)
    cache, table, lens, q = case
    home = torch.cuda.Stream()
    want = cache.attend(table, lens, q)
    torch.cuda.synchronize()
    graph, out = capture(case, home)
    later = [capture(split_case(5 + i), home) for i in range(2)]
    keep = (cache.k, cache.v, cache.k_scale, cache.v_scale, cache.status_word)     # (the codes stay the caller's to keep)
    del cache, case
    gc.collect()
    dirt = [torch.full((1 << 22,), 0xff, dtype=torch.uint8, device="cuda") for _ in range(16)]
    for _ in range(5):
        out.zero_()
        graph.replay()
        assert torch.equal(out, want)
        dirt[0].fill_(0x7f)
    assert len(later) == 2 and len(keep) == 5


def test_only_the_counters_have_to_be_zero():
    """A workspace made of memory that holds anything else."""
    cache, table, lens, q = split_case(3)
    want = cache.attend(table, lens, q)
    n, c = lib().dvi_paged_workspace_bytes(64), lib().dvi_paged_counter_bytes()
    assert 0 < c <= 4096 and c < n
    for fill in (0xff, 0x7f, 0x01):
        other, side = split_case(3)[0], torch.cuda.Stream()
        other.k.copy_(cache.k), other.v.copy_(cache.v), other.k_scale.copy_(cache.k_scale), other.v_scale.copy_(cache.v_scale)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            dirt = torch.full((n,), fill, dtype=torch.uint8, device="cuda")
            del dirt
            assert torch.equal(other.attend(table, lens, q), want)


def captured_nodes(stream):
    """How many nodes the graph has that `stream` is being captured into."""
    rt = ctypes.CDLL("libcudart.so.13")
    r, state, cid, graph, n = ctypes.byref, ctypes.c_int(), ctypes.c_uint64(), ctypes.c_void_p(), ctypes.c_size_t()
    assert rt.cudaStreamGetCaptureInfo(ctypes.c_void_p(stream.cuda_stream), r(state), r(cid), r(graph), None, None,
                                       None) == 0
    assert state.value == 1 and rt.cudaGraphGetNodes(graph, None, r(n)) == 0
    return n.value


@pytest.mark.parametrize("warm", [False, True])
def test_a_graph_clears_its_counters_once(warm):
    layers = [split_case(i) for i in range(6)]
    side = torch.cuda.Stream()
    if warm:
        with torch.cuda.stream(side):
            layers[0][0].attend(*layers[0][1:])
    want = [c.attend(t, n, q) for c, t, n, q in layers]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        outs = [c.attend(t, n, q) for c, t, n, q in layers]
        n = captured_nodes(side)
    assert n == len(layers) + 1          # a launch each, and the clearing
    for _ in range(3):
        for o in outs:
            o.zero_()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_caches_share_a_workspace():
    """A stream's calls run one after another: they use one workspace, whatever the cache, and it goes with the last."""
    gc.collect()
    start = torch.cuda.memory_allocated()
    layers = [split_case(i) for i in range(6)]
    before, size = torch.cuda.memory_allocated(), lib().dvi_paged_workspace_bytes(64)
    want = [c.attend(t, n, q) for c, t, n, q in layers]
    grown = torch.cuda.memory_allocated() - before - sum(w.numel() * 2 for w in want)
    assert grown < 2 * size, (grown, size)          # (the allocator rounds it up)
    for _ in range(3):
        assert all(torch.equal(c.attend(t, n, q), w) for (c, t, n, q), w in zip(layers, want))
    del layers, want
    gc.collect()
    assert torch.cuda.memory_allocated() - start < size
