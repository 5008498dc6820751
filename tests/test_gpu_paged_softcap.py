"""Score caps from far below the scores to far above them: c tanh(s / c) keeps the accuracy of the scores, and at caps
that no score comes near it is the score itself."""
import numpy as np
import pytest
import torch

import paged_ref as ref
from test_gpu_paged import check_attend, host, ints, make_cache, make_table

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cap", [1e-3, 0.3, 1.0, 8.0, 30.0, 50.0, 256.0, 257.0, 1e3, 1e4, 1e6, 1e8, 1e15, 9e29])
@pytest.mark.parametrize("rows", [1, 3, 40])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_caps(cap, rows, dtype):
    lens, n = [0, 61, 200], [rows] * 3
    cache = make_cache("int8", 64, 2, 16, 64, rows)
    check_attend(cache, make_table(lens, n, 16, 64, 4), lens, n, 6, dtype, seed=rows, softcap=cap)


@pytest.mark.parametrize("cap", [30.0, 1e8, 9e29])
@pytest.mark.parametrize("rows", [3, 40])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_mul", [1e-6, 1e-3, 20.0])
def test_caps_over_small_and_large_scores(cap, rows, dtype, q_mul):
    """Scores of 1e-5 to 1e3, with a window and a bias."""
    lens, n, D = [130], [rows], 128
    cache = make_cache("e4m3", 16, 2, 32, D, rows)
    q = (q_mul * torch.randn(rows, 6, D, device="cuda")).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    table, slopes = make_table(lens, n, 32, 16, 4), 2.0 ** -torch.arange(1, 7, device="cuda").float()
    out = cache.attend(ints(table), ints(lens), q, softcap=cap, window=100, slopes=slopes)
    kv = host(cache)
    o, mass, reach = ref.attend(kv, table, lens, [0, rows], q.double().cpu().numpy(), D ** -0.5, softcap=cap, window=100,
                                slopes=slopes.cpu().numpy())
    largest = np.abs(ref.values(kv["v"], "e4m3") * kv["v_scale"][:, :, None, None]).max()
    err = np.abs(out.double().cpu().numpy() - o)
    tol = ref.attend_bound(o, mass, reach, lens[0] + rows, D, dtype, largest)
    assert (err <= tol).all(), float((err / tol).max())


@pytest.mark.parametrize("rows", [3, 40])
def test_a_cap_out_of_reach_is_none(rows):
    """At a cap of 1e15 the capped score is the score: two results, each rounded by 2^-8 of itself, with weights rounded
    by 2^-11 of themselves and scores by a few 2^-24 of theirs (which 2^-12 more of the largest value covers)."""
    cache = make_cache("int8", 16, 2, 16, 64, 9)
    q = torch.randn(rows, 4, 64, device="cuda").bfloat16()
    table, lens = ints([list(range(16))]), ints([90])
    a = cache.attend(table, lens, q).float()
    b = cache.attend(table, lens, q, softcap=1e15).float()
    most = cache.read(table, ints([0]), 90 + rows, dtype=torch.float32)[1].abs().amax()
    assert ((a - b).abs() <= 2.0 ** -7 * a.abs() + (2.0 ** -10 + 2.0 ** -12) * most).all()
