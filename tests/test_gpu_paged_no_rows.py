"""Rows that a max_rows of 0 shuts out are dropped like any others past max_rows: flagged."""
import numpy as np
import pytest
import torch

from test_gpu_paged import host, ints, make_cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("call", ["append", "attend", "read"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_no_rows_allowed(call, dtype):
    cache = make_cache("int8", 8, 2, 16, 64, 1)
    table, lens = ints(np.arange(8).reshape(2, 4)), ints([5, 6])
    q, kv = torch.randn(8, 4, 64, device="cuda").to(dtype), torch.randn(8, 2, 64, device="cuda").to(dtype)
    before = host(cache)
    for start, flags in (([0, 7, 8], ["KV_FULL"]), ([0, 0, 0], [])):
        out = torch.full_like(q, 7)
        if call == "append":
            cache.append(table, lens, kv, kv, q=q, q_out=out, row_start=ints(start), max_rows=0)
        elif call == "attend":
            cache.attend(table, lens, q, row_start=ints(start), max_rows=0, out=out)
        else:
            cache.read(table, lens, 8, row_start=ints(start), max_rows=0, dtype=dtype)
        assert cache.status() == flags
        assert (out == 7).all()
    assert all((host(cache)[x] == before[x]).all() for x in ("k", "v", "k_scale", "v_scale"))
