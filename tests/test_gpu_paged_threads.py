"""attend from several host threads: on one stream their calls follow each other whole, also where a call is two launches
side by side, and on streams of their own they do not meet."""
import ctypes
import threading

import numpy as np
import pytest
import torch

from paper_2510_05421_gb300 import lib
from paper_2510_05421_gb300.paged import PagedBatchC, PagedOptionsC
from test_gpu_paged import ints, make_cache, make_table

pytestmark = pytest.mark.gpu


def mixed(seed):
    """A prompt chunk beside tokens over long contexts: two launches, both of them splitting and joining."""
    P, H, D, lens, rows = 64, 2, 64, [500, 9000, 7000], [150, 2, 3]
    pages = sum(-(-(a + b) // P) for a, b in zip(lens, rows))
    cache = make_cache("int8", pages, H, P, D, seed)
    table = ints(make_table(lens, rows, P, pages, seed))
    start = ints(np.concatenate([[0], np.cumsum(rows)]))
    return cache, table, ints(lens), start, torch.randn(sum(rows), 8, D, device="cuda").bfloat16()


def run_threads(bodies):
    failed = []

    def guarded(body):
        try:
            body()
        except Exception as e:      # noqa: BLE001
            failed.append(e)

    threads = [threading.Thread(target=guarded, args=(b,)) for b in bodies]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed


def test_c_calls_of_one_stream():
    """Through the C entry, with the one workspace that the calls of a stream need."""
    n_threads, times, D = 4, 60, 64
    cases = [mixed(i) for i in range(n_threads)]
    want = [c.attend(t, n, q, row_start=s, max_rows=150) for c, t, n, s, q in cases]
    ws = torch.zeros(lib().dvi_paged_workspace_bytes(D), dtype=torch.uint8, device="cuda")
    out = [[torch.zeros_like(c[4]) for _ in range(times)] for c in cases]
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()

    def body(i):
        cache, table, lens, start, q = cases[i]
        batch = PagedBatchC(3, table.shape[1], q.shape[0], 150, table.data_ptr(), lens.data_ptr(), start.data_ptr(),
                            cache.status_word.data_ptr())
        options, r = PagedOptionsC(8, D ** -0.5, 0.0, 0, None), ctypes.byref
        for o in out[i]:
            rc = lib().dvi_paged_attend(r(cache._c), r(batch), r(options), 1, q.data_ptr(), 8 * D, o.data_ptr(), 8 * D,
                                        ws.data_ptr(), ws.numel(), stream.cuda_stream)
            assert rc == 0

    run_threads([lambda i=i: body(i) for i in range(n_threads)])
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for outs, w in zip(out, want) for o in outs)
    assert all(c[0].status() == [] for c in cases)


@pytest.mark.parametrize("own_streams", [False, True])
def test_python_calls(own_streams):
    n_threads, times = 4, 40
    cases = [mixed(10 + i) for i in range(n_threads)]
    want = [c.attend(t, n, q, row_start=s, max_rows=150) for c, t, n, s, q in cases]
    streams = [torch.cuda.Stream() for _ in range(n_threads if own_streams else 1)] * (1 if own_streams else n_threads)
    got = [[] for _ in cases]
    torch.cuda.synchronize()

    def body(i):
        cache, table, lens, start, q = cases[i]
        with torch.cuda.stream(streams[i]):
            for _ in range(times):
                got[i].append(cache.attend(table, lens, q, row_start=start, max_rows=150))

    run_threads([lambda i=i: body(i) for i in range(n_threads)])
    torch.cuda.synchronize()
    assert all(len(g) == times and all(torch.equal(o, w) for o in g) for g, w in zip(got, want))
