"""attend with fewer live rows than the call has room for: a buffer of fixed size with its row starts on the device (what
a captured graph replays), and a C call whose max_rows is only an upper bound.  Every live row is written, whichever
kernel's the row counts are, and no other row is touched."""
import ctypes

import numpy as np
import pytest
import torch

import paged_ref as ref
from paper_2510_05421_gb300 import lib
from paper_2510_05421_gb300.paged import PagedBatchC, PagedOptionsC
from test_gpu_paged import host, ints, make_cache, make_table

pytestmark = pytest.mark.gpu
TD = {"bf16": torch.bfloat16, "f32": torch.float32}


def live_rows_are_right(cache, table, lens, starts, q, out, dtype):
    """out: filled with 7 before the call; rows from starts[-1] on are nobody's."""
    D, n = cache.head_dim, int(starts[-1])
    o, mass, reach = ref.attend(host(cache), np.asarray(table), lens, starts, q[:n].double().cpu().numpy(), D ** -0.5)
    keys = max(a + c for a, c in zip(lens, np.diff(starts)))
    err = np.abs(out[:n].double().cpu().numpy() - o)
    tol = ref.attend_bound(o, mass, reach, keys, D, dtype)
    assert (err <= tol).all(), float((err / tol).max())
    assert (out[n:] == 7).all()
    assert cache.status() == []


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("group", [1, 4])
@pytest.mark.parametrize("rows", [[0], [1], [3], [8], [9], [32], [33], [64], [3, 1], [0, 40], [64, 0], [2, 60]])
def test_buffer_with_room(rows, group, D, dtype):
    B, H, P = len(rows), 2, 32
    room = 64 * B
    lens = [70, 129][:B]
    cache = make_cache("int8", 16, H, P, D, sum(rows) + group)
    table = make_table(lens, [64] * B, P, 16, 3)
    starts = np.concatenate([[0], np.cumsum(rows)])
    g = torch.Generator(device="cuda")
    g.manual_seed(sum(rows))
    q = (1.5 * torch.randn(room, group * H, D, device="cuda", generator=g)).to(TD[dtype])
    for bound in (None, 64):
        out = torch.full_like(q, 7)
        cache.attend(ints(table), ints(lens), q, row_start=ints(starts), max_rows=bound, out=out)
        live_rows_are_right(cache, table, lens, starts, q, out, dtype)


@pytest.mark.parametrize("B,rows,G,bound", [(64, 1, 2, 64), (8, 1, 8, 8), (3, 5, 1, 500), (1, 3, 4, 1000), (2, 40, 1, 200)])
def test_loose_bound_without_row_starts(B, rows, G, bound):
    """The C entry takes any max_rows from n_rows / n_seqs on."""
    H, P, D = 2, 16, 64
    lens = [33 + b % 50 for b in range(B)]
    pages = sum(-(-(a + rows) // P) for a in lens)
    cache = make_cache("e4m3", pages, H, P, D, B)
    table = make_table(lens, [rows] * B, P, pages, 4)
    q = torch.randn(B * rows, G * H, D, device="cuda").bfloat16()
    out = torch.full_like(q, 7)
    tab, ln, ws = ints(table), ints(lens), torch.zeros(lib().dvi_paged_workspace_bytes(D), dtype=torch.uint8, device="cuda")
    batch = PagedBatchC(B, tab.shape[1], B * rows, bound, tab.data_ptr(), ln.data_ptr(), None, cache.status_word.data_ptr())
    options = PagedOptionsC(G * H, D ** -0.5, 0.0, 0, None)
    r = ctypes.byref
    rc = lib().dvi_paged_attend(r(cache._c), r(batch), r(options), 1, q.data_ptr(), G * H * D, out.data_ptr(), G * H * D,
                                ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream)
    assert rc == 0
    live_rows_are_right(cache, table, lens, np.arange(B + 1) * rows, q, out, "bf16")
