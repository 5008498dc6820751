"""The 8-bit paged KV cache (append, attend, read) against plain 64-bit
restatements, over page sizes, formats, head groups, ragged rows, lengths
around every tile and page boundary, holes, masks that leave a row empty,
garbage behind the last row, strides and streams.

Tolerances follow from the formats.  Attend: with A = sum p |v| of a row, S =
the largest sum |q k| scale, n keys: a score is off by at most S times
(head_dim + 8) 2^-23 (f32 products and sums that may truncate), which moves
the result by at most twice that times A; a weight's f16 rounding is 2^-11 of
it (f32 queries: two f16 numbers, 2^-21), the sums of n weights (n / 16 + 64)
2^-23 of A, and a bf16 result (8 significant bits) is
rounded by 2^-8 of itself."""
import numpy as np
import pytest
import torch

import paged_ref as ref
from paper_2510_05421_gb300 import PagedCache, rotary_table

pytestmark = pytest.mark.gpu
CODE = {"int8": torch.int8, "e4m3": torch.uint8}
TD = {"bf16": torch.bfloat16, "f32": torch.float32}


def make_cache(fmt, n_pages, H, P, D, seed, scale_lo=0.005, scale_hi=0.02):
    """A cache whose every row (also those that nobody owns) holds random codes."""
    g = np.random.default_rng(seed)
    codes = []
    for _ in range(2):
        c = g.integers(-127, 128, (n_pages, H, P, D)).astype(np.int8)
        if fmt == "e4m3":
            c = g.integers(0, 256, (n_pages, H, P, D)).astype(np.uint8)
            c[(c & 0x7f) == 0x7f] = 3
            c[(c & 0x7f) > 0x70] &= 0xbf      # magnitudes up to 3.75 and then some
        codes.append(torch.from_numpy(c).cuda())
    sc = [torch.from_numpy(g.uniform(scale_lo, scale_hi, (n_pages, H)).astype(np.float32)).cuda() for _ in range(2)]
    return PagedCache(codes[0], codes[1], sc[0], sc[1], fmt=fmt)


def host(cache):
    return dict(k=cache.k.cpu().numpy(), v=cache.v.cpu().numpy(), k_scale=cache.k_scale.cpu().numpy(),
                v_scale=cache.v_scale.cpu().numpy(), fmt=cache.fmt)


def make_table(lens, rows, P, n_pages, seed, extra=0):
    need = [-(-(a + b) // P) for a, b in zip(lens, rows)]
    order = np.random.default_rng(seed).permutation(n_pages)
    assert sum(need) <= n_pages
    t = np.full((len(lens), max(need) + extra), -1, np.int32)
    at = 0
    for b, m in enumerate(need):
        t[b, :m] = order[at:at + m]
        at += m
    return t


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32).cuda()


def check_attend(cache, table, lens, rows, Hq, dtype, seed=0, scale=None, q=None, **opt):
    D = cache.head_dim
    n = sum(rows)
    starts = np.concatenate([[0], np.cumsum(rows)])
    if q is None:
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        q = (1.5 * torch.randn(n, Hq, D, device="cuda", generator=g)).to(TD[dtype])
    slopes = opt.get("slopes")
    out = cache.attend(ints(table), ints(lens), q, scale=scale, row_start=ints(starts), max_rows=max(rows), **opt)
    torch.cuda.synchronize()
    ro = dict(opt, slopes=None if slopes is None else slopes.cpu().numpy())
    o, mass, reach = ref.attend(host(cache), np.asarray(table), lens, starts, q.double().cpu().numpy(),
                                D ** -0.5 if scale is None else scale, **ro)
    keys = max(a + b for a, b in zip(lens, rows))
    tol = mass * (2 * reach[..., None] * (D + 8) * 2.0 ** -23 + (keys / 16 + 64) * 2.0 ** -23 +
                  (2.0 ** -11 if dtype == "bf16" else 2.0 ** -21)) + 1e-30
    if dtype == "bf16":
        tol = tol + np.abs(o) * 2.0 ** -8
    err = np.abs(out.double().cpu().numpy() - o)
    assert (err <= tol).all(), (float((err / tol).max()), np.argwhere(err > tol)[:3])
    return out


# ---------------------------------------------------------------- attend

@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("P", [16, 32, 64, 128])
def test_attend_lengths(D, fmt, dtype, P):
    """One token over contexts around every boundary, one after another in a ragged batch."""
    lens = [0, 1, 14, 15, 16, 17, 31, 32, 47, 63, 64, 95, 127, 128, 129, 255, 300]
    rows = [1] * len(lens)
    cache = make_cache(fmt, 3 * sum(-(-(a + 1) // P) for a in lens) // 2, 2, P, D, P + D)
    table = make_table(lens, rows, P, cache.n_pages, 1, extra=1)
    check_attend(cache, table, lens, rows, 4, dtype)
    assert cache.status() == []


@pytest.mark.parametrize("group", [1, 2, 3, 4, 5, 7, 8, 16])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_groups_and_row_counts(group, dtype):
    """Ragged row counts, none among them, on both sides of every tile width."""
    rows = [1, 2, 0, 5, 9, 3, 17, 33]
    lens = [70, 0, 12, 3, 100, 200, 41, 7]
    cache = make_cache("int8", 64, 2, 32, 64, group)
    table = make_table(lens, rows, 32, 64, 2)
    check_attend(cache, table, lens, rows, 2 * group, dtype, seed=group)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("D,group,rows", [(128, 2, 150), (64, 4, 131), (128, 1, 257), (64, 8, 64), (128, 3, 90),
                                          (128, 7, 61)])
def test_attend_prompt_chunks(fmt, D, group, rows):
    """Many rows of a sequence, behind a prefix and from an empty cache, beside single tokens."""
    lens, n = [77, 0, 130, 0], [rows, rows - 3, 1, 128]
    cache = make_cache(fmt, 40, 2, 64, D, rows)
    table = make_table(lens, n, 64, 40, 3)
    check_attend(cache, table, lens, n, 2 * group, "bf16", seed=rows)


@pytest.mark.parametrize("B,H,ctx,rows,page,opt", [(40, 48, 0, 40, 16, dict()), (3, 40, 500, 300, 64, dict()),
                                                   (1, 39, 1500, 130, 128, dict()), (5, 32, 40, 270, 32, dict(window=150)),
                                                   (1, 1, 3000, 200, 64, dict()), (2, 77, 900, 131, 64, dict(softcap=8.0))])
def test_attend_prompts_are_shared(B, H, ctx, rows, page, opt):
    """Prompt chunks in more and fewer units than SMs, of even and uneven lengths, cut by shares and by splits;
    twice, as what the first call leaves in the workspace is the second's to find."""
    lens = [ctx + 37 * (b % 5) for b in range(B)]
    n = [max(rows - 29 * (b % 3), 5) for b in range(B)]
    pages = sum(-(-(a + r) // page) for a, r in zip(lens, n))
    cache = make_cache("int8", pages, H, page, 64, B)
    table = make_table(lens, n, page, pages, 5)
    for seed in (1, 2):
        check_attend(cache, table, lens, n, H, "bf16", seed=seed, **opt)


@pytest.mark.parametrize("rows", [1, 6, 40, 140])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("opt", [dict(softcap=20.0), dict(window=1), dict(window=33), dict(window=100, softcap=5.0),
                                 dict(slopes=True), dict(slopes=True, softcap=30.0, window=64)])
def test_attend_options(rows, dtype, opt):
    lens, n = [0, 61, 200], [rows] * 3
    if dtype == "f32" and rows > 100:
        n = [rows, 1, 2]
    opt = dict(opt)
    if opt.get("slopes"):
        opt["slopes"] = (2.0 ** -torch.arange(1, 7, device="cuda").float())
    cache = make_cache("int8", 64, 2, 16, 64, rows)
    check_attend(cache, make_table(lens, n, 16, 64, 4), lens, n, 6, dtype, seed=rows, **opt)


@pytest.mark.parametrize("rows", [1, 4, 70])
def test_attend_pages_not_held(rows):
    """Holes: at the front, in the middle, and everything but the row's own page; a row with no page at
    all, or whose window has none, gets zeros."""
    P, lens, n = 16, [90, 90, 90, 90], [rows] * 4
    cache = make_cache("e4m3", 64, 2, P, 64, 5)
    table = make_table(lens, n, P, 64, 5)
    table[0, :3] = -1
    table[1, 2:5] = -7
    table[2, :] = -1
    table[3, 1:] = -1
    out = check_attend(cache, table, lens, n, 4, "bf16")
    assert (out[2 * rows:3 * rows] == 0).all()
    w = check_attend(cache, table, lens, n, 4, "bf16", window=40)
    assert (w[3 * rows:4 * rows] == 0).all()
    assert cache.status() == []


@pytest.mark.parametrize("rows", [3, 80])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_attend_reads_nothing_behind_the_last_row(rows, fmt):
    """Codes past a sequence's rows are NaN (e4m3) or extreme, scales of unused pages NaN and infinite:
    no result changes, bit for bit."""
    P, lens, n = 16, [33, 0, 20], [rows] * 3
    cache = make_cache(fmt, 40, 2, P, 64, 6)
    table = make_table(lens, n, P, 40, 6, extra=2)
    q = torch.randn(3 * rows, 4, 64, device="cuda").bfloat16()
    a = cache.attend(ints(table), ints(lens), q)
    used = set()
    for b in range(3):
        end = lens[b] + rows
        for s in range(-(-end // P)):
            used.add(int(table[b, s]))
        page, off = int(table[b, (end - 1) // P]), (end - 1) % P + 1
        for pool in (cache.k, cache.v):
            pool[page, :, off:] = 0x7f
    for p in range(40):
        if p not in used:
            cache.k_scale[p], cache.v_scale[p] = float("nan"), float("inf")
            cache.k[p] = 0x7f
            cache.v[p] = 0x7f
    table[table < 0] = [p for p in range(40) if p not in used][0]
    b = cache.attend(ints(table), ints(lens), q)
    assert torch.equal(a, b)


def test_attend_bad_query_stays_in_its_row():
    cache = make_cache("int8", 16, 2, 16, 64, 7)
    lens, table = ints([40]), ints(np.arange(16)[None])
    q = torch.randn(6, 4, 64, device="cuda")
    good = cache.attend(table, lens, q)
    q[2, 1, 5], q[4, 3, 0] = float("nan"), float("inf")
    bad = cache.attend(table, lens, q)
    hit = torch.zeros(6, 4, dtype=torch.bool, device="cuda")
    hit[2, 1] = hit[4, 3] = True
    assert torch.equal(good[~hit], bad[~hit])
    assert not torch.isfinite(bad[hit]).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("k_mul,v_mul,q_mul", [(1e-20, 1e-12, 1e18), (1e6, 1e9, 1e-7), (1.0, 1e-15, 1e-30)])
def test_attend_extreme_scales(dtype, k_mul, v_mul, q_mul):
    """Page scales and queries far outside f16's range, and pages of one sequence that differ by 1e6."""
    cache = make_cache("int8", 32, 2, 16, 64, 8, 0.5, 1.0)
    cache.k_scale.mul_(k_mul)
    cache.v_scale.mul_(v_mul)
    cache.v_scale[::2] *= 1e-6
    lens, rows = [200, 77], [5, 5]
    q = (q_mul * torch.randn(10, 4, 64, device="cuda")).to(TD[dtype])
    check_attend(cache, make_table(lens, rows, 16, 32, 8), lens, rows, 4, dtype, q=q, scale=0.003)


@pytest.mark.parametrize("B,ctx,rows,Hq,H", [(1, 5000, 1, 8, 8), (1, 5000, 6, 4, 1), (40, 600, 1, 4, 4),
                                             (3, 2100, 30, 8, 2)])
def test_attend_work_is_split_and_joined(B, ctx, rows, Hq, H):
    """Shares that cut groups and hold several of them; the same call gives the same bits."""
    lens = [ctx - 13 * b for b in range(B)]
    n = [rows] * B
    P = 64
    pages = sum(-(-(a + rows) // P) for a in lens)
    cache = make_cache("int8", pages, H, P, 64, B)
    table = make_table(lens, n, P, pages, 9)
    out = check_attend(cache, table, lens, n, Hq, "bf16", seed=B)
    q = torch.randn(B * rows, Hq, 64, device="cuda").bfloat16()
    first = cache.attend(ints(table), ints(lens), q)
    for _ in range(20):
        assert torch.equal(first, cache.attend(ints(table), ints(lens), q))
    assert out.shape == first.shape


def test_attend_offsets_past_32_bits():
    """Pages whose codes lie more than 2^32 bytes into the pool."""
    H, P, D = 8, 128, 128
    n_pages = (2 ** 32 // (H * P * D)) + 40
    k = torch.zeros(n_pages, H, P, D, dtype=torch.int8, device="cuda")
    v = torch.zeros(n_pages, H, P, D, dtype=torch.int8, device="cuda")
    sc = torch.full((n_pages, H), 0.01, device="cuda")
    big = PagedCache(k, v, sc, sc.clone())
    small = make_cache("int8", 8, H, P, D, 10)
    at = torch.arange(n_pages - 8, n_pages, device="cuda")
    for x, y in ((big.k, small.k), (big.v, small.v), (big.k_scale, small.k_scale), (big.v_scale, small.v_scale)):
        x[at] = y
    lens = ints([900])
    for rows in (2, 70):
        q = torch.randn(rows, 16, D, device="cuda").bfloat16()
        a = big.attend(at.to(torch.int32)[None].contiguous(), lens, q)
        b = small.attend(ints(np.arange(8)[None]), lens, q)
        assert torch.equal(a, b)
    kn, vn = torch.randn(3, H, D, device="cuda"), torch.randn(3, H, D, device="cuda")
    big.append(at.to(torch.int32)[None].contiguous(), lens, kn, vn)
    small.append(ints(np.arange(8)[None]), lens, kn, vn)
    assert torch.equal(big.k[at], small.k) and torch.equal(big.v_scale[at], small.v_scale)
    ra = big.read(at.to(torch.int32)[None].contiguous(), lens, 3)
    rb = small.read(ints(np.arange(8)[None]), lens, 3)
    assert torch.equal(ra[0], rb[0]) and torch.equal(ra[1], rb[1])


def test_attend_out_of_range_device_values_are_flagged():
    """Negative lengths, lengths past the table, row starts past the rows and entries past the pool stay
    inside the buffers and are reported."""
    cache = make_cache("int8", 8, 2, 16, 64, 11)
    q = torch.randn(8, 4, 64, device="cuda").bfloat16()
    kv = torch.randn(8, 2, 64, device="cuda")
    good = ints(np.arange(8).reshape(2, 4))
    for table, lens, start in ((good, [-5, 3], [0, 4, 8]), (good, [2 ** 31 - 1, 70], [0, 4, 8]),
                               (good, [5, 6], [0, 4, 99]), (good, [5, 6], [0, -3, 8]), (good, [5, 6], [7, 2, 8]),
                               (ints([[1, 8, 2, 3], [900, 5, 6, 7]]), [30, 9], [0, 4, 8])):
        cache.status()
        out = cache.attend(table, ints(lens), q, row_start=ints(start))
        cache.read(table, ints(lens), 8, row_start=ints(start))
        assert "KV_FULL" in cache.status(), (lens, start)
        cache.append(table, ints(lens), kv, kv, row_start=ints(start))
        assert "KV_FULL" in cache.status(), (lens, start)
        assert out.shape == q.shape


@pytest.mark.parametrize("start", [[0, 900, 300, 1000], [700, 100, 900, 1000], [0, -50, 1200, 1000], [1000, 0, 0, 0]])
def test_row_starts_that_do_not_ascend_stay_inside(start):
    """Prompt-sized calls whose row starts fall: flagged, and no row outside the call is read or written."""
    cache = make_cache("int8", 60, 2, 64, 64, 13)
    table, lens = ints(np.arange(60).reshape(3, 20)), ints([0, 64, 100])
    room = torch.full((1400, 8, 64), 7.0, device="cuda").bfloat16()
    q = torch.randn(1400, 8, 64, device="cuda").bfloat16()
    cache.attend(table, lens, q[200:1200], row_start=ints(start), out=room[200:1200])
    assert "KV_FULL" in cache.status()
    assert (room[:200] == 7).all() and (room[1200:] == 7).all()
    kv = torch.randn(1000, 2, 64, device="cuda")
    cache.append(table, lens, kv, kv, row_start=ints(start))
    cache.read(table, lens, 1000, row_start=ints(start))
    assert "KV_FULL" in cache.status()


@pytest.mark.parametrize("rows", [2, 50])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_huge_scores(rows, dtype):
    """Scores around -6e33, where f32 holds no difference between them: the result is still a mean of the
    values that the row sees (weighted somehow), so within their range."""
    cache = make_cache("int8", 8, 1, 16, 64, 14)
    cache.k[:] = 100
    cache.k_scale[:] = 1e15
    q = torch.full((rows, 2, 64), -1e17, device="cuda").to(TD[dtype])
    lens = ints([40])
    out = cache.attend(ints(np.arange(8)[None]), lens, q, scale=0.01).float()
    _, v = cache.read(ints(np.arange(8)[None]), ints([0]), 40 + rows, dtype=torch.float32)
    for r in range(rows):
        lo, hi = v[:41 + r, 0].amin(0), v[:41 + r, 0].amax(0)
        # rounded by 2^-8 of itself (bf16), and the means by less than 2^-10 of the largest value
        slack = (lo.abs() + hi.abs()) * (2.0 ** -8 + 2.0 ** -10)
        assert torch.isfinite(out[r]).all() and (out[r] >= lo - slack).all() and (out[r] <= hi + slack).all()


@pytest.mark.parametrize("rows", [1, 5, 40, 150])
@pytest.mark.parametrize("opt", [dict(), dict(window=20), dict(softcap=10.0)])
def test_attend_zero_queries_and_keys(rows, opt):
    """Padding: queries of zeros over pages whose keys are zeros (a scale of 2^-80): a score's factor is below
    what f32 holds, and positions behind a row stay out of it all the same."""
    cache = make_cache("int8", 16, 2, 16, 64, 18)
    cache.k[:8] = 0
    cache.k_scale[:8] = 2.0 ** -80
    q = torch.zeros(rows, 4, 64, device="cuda").bfloat16()
    check_attend(cache, np.arange(16)[None], [33], [rows], 4, "bf16", q=q, **opt)


@pytest.mark.parametrize("rows", [3, 40])
def test_attend_window_past_every_position(rows):
    """A window of 2^31 - 1 positions is none."""
    cache = make_cache("e4m3", 8, 2, 32, 64, 15)
    q = torch.randn(rows, 4, 64, device="cuda").bfloat16()
    a = cache.attend(ints(np.arange(8)[None]), ints([100]), q)
    assert torch.equal(a, cache.attend(ints(np.arange(8)[None]), ints([100]), q, window=2 ** 31 - 1))


def test_graph_of_a_mixed_batch():
    """Prompts, blocks and tokens in one captured call (two launches side by side), replayed between writes to
    its inputs by the surrounding kernels."""
    cache = make_cache("int8", 40, 2, 64, 128, 16)
    lens, n = [77, 0, 130], [150, 3, 1]
    table, start = ints(make_table(lens, n, 64, 40, 3)), ints(np.concatenate([[0], np.cumsum(n)]))
    q = torch.zeros(154, 4, 128, device="cuda").bfloat16()
    fresh = [torch.randn(154, 4, 128, device="cuda").bfloat16() for _ in range(8)]
    want = [cache.attend(table, ints(lens), x, row_start=start, max_rows=150).clone() for x in fresh]
    ln = ints(lens)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        cache.attend(table, ln, q, row_start=start, max_rows=150)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = cache.attend(table, ln, q, row_start=start, max_rows=150) * 1
    for x, w in zip(fresh, want):
        q.copy_(x)
        graph.replay()
        assert torch.equal(out, w)


def test_attend_more_rows_than_max_rows_are_flagged():
    cache = make_cache("int8", 8, 2, 16, 64, 12)
    q = torch.randn(8, 4, 64, device="cuda").bfloat16()
    table, lens = ints(np.arange(8).reshape(2, 4)), ints([5, 6])
    cache.attend(table, lens, q, row_start=ints([0, 7, 8]), max_rows=4)
    assert cache.status() == ["KV_FULL"]


# ---------------------------------------------------------------- append

def check_append(cache, table, lens, rows, k, v, rotary, before):
    """The cache after an append against the 64-bit definition from the state `before` it."""
    fmt, P, H = cache.fmt, cache.page_tokens, cache.n_kv_heads
    after = host(cache)
    starts = np.concatenate([[0], np.cumsum(rows)])
    rot = None if rotary is None else rotary.cpu().numpy()
    k, v = k.double().cpu().numpy(), v.double().cpu().numpy()
    touched = {}
    for b in range(len(lens)):
        for r in range(starts[b], starts[b + 1]):
            p = lens[b] + r - starts[b]
            touched.setdefault((b, p // P), []).append((p, r))
    mine = set()
    for (b, slot), items in touched.items():
        page = int(table[b, slot])
        mine.add(page)
        held = max(0, lens[b] - slot * P)
        for name, x in (("k", k), ("v", v)):
            fresh = np.stack([ref.rotate(x[r], p, rot if name == "k" else None) for p, r in items], 1)   # [H, m, D]
            sc = np.maximum(np.abs(fresh).max((1, 2)) / ref.TOP[fmt], ref.MIN_SCALE)
            was = before[name + "_scale"][page].astype(np.float64)
            if held:
                sc = np.maximum(sc, was)
            got_sc = after[name + "_scale"][page].astype(np.float64)
            assert np.allclose(got_sc, sc, rtol=2.0 ** -21, atol=0)
            codes = ref.values(after[name][page], fmt)                                                    # [H, P, D]
            # a value is within half a step of the true one (and the f32 arithmetic's 2^-20)
            want = fresh / sc[:, None, None]
            new = codes[:, [p % P for p, _ in items]]
            half = 0.5 * np.maximum(ref.step_of(want, fmt), ref.step_of(new, fmt))
            assert (np.abs(new - want) <= half + np.abs(want) * 2.0 ** -20 + 1e-30).all()
            old = ref.values(before[name][page], fmt)[:, :held]
            grown = (sc > was * (1 + 2.0 ** -22)) if held else np.zeros(H, bool)
            for h in range(H):
                now = codes[h, :held]
                if held and grown[h]:
                    true = old[h] * (was[h] / sc[h])
                    half = 0.5 * np.maximum(ref.step_of(true, fmt), ref.step_of(now, fmt))
                    assert (np.abs(now - true) <= half + np.abs(true) * 2.0 ** -20).all()
                elif held and sc[h] == was[h]:
                    assert (now == old[h]).all()
            rest = [i for i in range(P) if i >= held and i not in {p % P for p, _ in items}]
            assert (after[name][page][:, rest] == before[name][page][:, rest]).all()
    others = [p for p in range(cache.n_pages) if p not in mine]
    for name in ("k", "v", "k_scale", "v_scale"):
        assert (after[name][others] == before[name][others]).all()


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("P", [16, 32, 64, 128])
@pytest.mark.parametrize("D,rot", [(64, 64), (64, 0), (128, 128), (128, 32), (64, 48)])
def test_append(fmt, dtype, P, D, rot):
    lens = [0, 5, P - 1, P, 2 * P + 3, 17, 40]
    rows = [1, 4, 3, P + 2, 2 * P, 0, 7]
    H, Hq = 3, 6
    n = sum(rows)
    cache = make_cache(fmt, 32, H, P, D, P)
    table = make_table(lens, rows, P, 32, P)
    g = torch.Generator(device="cuda")
    g.manual_seed(P + D + rot)
    qkv = torch.randn(n, Hq + 2 * H, D, device="cuda", generator=g).to(TD[dtype])
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
    v[3] = 0
    rotary = rotary_table(4 * P + 64, rot) if rot else None
    before = host(cache)
    starts = np.concatenate([[0], np.cumsum(rows)])
    args = (ints(table), ints(lens), k, v)
    kw = dict(rotary=rotary, row_start=ints(starts), max_rows=max(rows))
    q2 = cache.append(*args, q=q, **kw)
    assert cache.status() == []
    check_append(cache, table, lens, rows, k, v, rotary, before)
    for b in range(len(lens)):
        for r in range(starts[b], starts[b + 1]):
            want = ref.rotate(q[r].double().cpu().numpy(), lens[b] + r - starts[b],
                              None if rotary is None else rotary.cpu().numpy())
            size = np.abs(q[r].double().cpu().numpy()).max()
            tol = np.abs(want) * (2.0 ** -8 if dtype == "bf16" else 0) + size * 2.0 ** -21
            assert (np.abs(q2[r].double().cpu().numpy() - want) <= tol).all()
    # again: the scales have what they need, so nothing moves
    once = host(cache)
    cache.append(*args, **kw)
    twice = host(cache)
    assert all((once[x] == twice[x]).all() for x in ("k", "v", "k_scale", "v_scale"))


def test_append_in_place_queries_and_strides():
    """q_out = q inside the projection's output, rows 16-byte aligned but far apart."""
    H, D, n = 2, 64, 5
    cache, other = make_cache("int8", 4, H, 16, D, 1), make_cache("int8", 4, H, 16, D, 1)
    wide = torch.randn(n, 1000, device="cuda").bfloat16()
    q = wide[:, 8:8 + 4 * D].view(n, 4, D)
    k = wide[:, 400:400 + H * D].view(n, H, D)
    v = wide[:, 600:600 + H * D].view(n, H, D)
    rotary = rotary_table(64, D)
    table, lens = ints([[0, 1]]), ints([10])
    want = other.append(table, lens, k.contiguous(), v.contiguous(), q=q.contiguous(), rotary=rotary)
    kk, vv = k.clone(), v.clone()
    got = cache.append(table, lens, k, v, q=q, q_out=q, rotary=rotary)
    assert got.data_ptr() == q.data_ptr() and torch.equal(got, want)
    assert torch.equal(k, kk) and torch.equal(v, vv)
    assert torch.equal(cache.k, other.k) and torch.equal(cache.v_scale, other.v_scale)
    out = torch.zeros(n, 600, device="cuda").bfloat16()
    o = out[:, 24:24 + 4 * D].view(n, 4, D)
    cache.attend(table, lens, q, out=o)
    assert torch.equal(o, cache.attend(table, lens, want))
    assert (out[:, :24] == 0).all() and (out[:, 24 + 4 * D:] == 0).all()


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_append_not_finite(fmt):
    """NaN is stored as 0, infinities as the largest code, other values as without them."""
    cache = make_cache(fmt, 4, 2, 16, 64, 2)
    k, v = torch.randn(4, 2, 64, device="cuda"), torch.randn(4, 2, 64, device="cuda")
    k[1, 0, 3], k[2, 0, 7], v[0, 1, 0], v[3, 1, 9] = float("nan"), float("inf"), float("-inf"), float("nan")
    table, lens = ints([[2]]), ints([0])
    cache.append(table, lens, k, v)
    assert cache.status() == ["NONFINITE"]
    kr, vr = cache.read(table, lens, 4, dtype=torch.float32)
    top = ref.TOP[fmt]
    assert kr[1, 0, 3] == 0 and vr[3, 1, 9] == 0
    assert kr[2, 0, 7] == cache.k_scale[2, 0] * top and vr[0, 1, 0] == -cache.v_scale[2, 1] * top
    clean = torch.where(torch.isfinite(k), k, 0.0)
    assert torch.allclose(cache.k_scale[2], clean.abs().amax((0, 2)) / top, rtol=1e-6)
    cache.append(table, lens, torch.zeros_like(k), torch.zeros_like(v))
    kr, vr = cache.read(table, lens, 4, dtype=torch.float32)
    assert (kr == 0).all() and (vr == 0).all()
    assert cache.status() == []


def test_append_drops_rows_without_a_page():
    cache = make_cache("int8", 6, 2, 16, 64, 3)
    before = host(cache)
    k = torch.randn(40, 2, 64, device="cuda")
    cache.append(ints([[3, -1]]), ints([10]), k, k)         # 6 rows on page 3, 16 on no page, 18 past the table
    assert cache.status() == ["KV_FULL"]
    after = host(cache)
    assert (after["k"][[0, 1, 2, 4, 5]] == before["k"][[0, 1, 2, 4, 5]]).all()
    kr, _ = cache.read(ints([[3, -1]]), ints([10]), 22, dtype=torch.float32)
    assert torch.allclose(kr[:6], k[:6], atol=float(cache.k_scale[3].max()))
    assert (kr[6:] == 0).all()


def test_append_rotary_shorter_than_the_positions_is_flagged():
    cache = make_cache("int8", 4, 2, 16, 64, 3)
    k = torch.randn(4, 2, 64, device="cuda")
    cache.append(ints([[0, 1]]), ints([10]), k, k, rotary=rotary_table(12, 64))
    assert cache.status() == ["KV_FULL"]


def test_rollback_and_append_again():
    """Rows past a lowered length are overwritten: what is read afterwards is the new rows'."""
    cache = PagedCache.create(8, 2, 64, page_tokens=16)
    table = ints(np.arange(8)[None])
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    k = torch.randn(50, 2, 64, device="cuda", generator=g)
    cache.append(table, ints([0]), k[:20], k[:20])
    cache.append(table, ints([20]), 3 * k[20:26], 3 * k[20:26])       # a drafted block, rejected after two rows
    cache.append(table, ints([22]), k[30:36], k[30:36])
    kr, vr = cache.read(table, ints([0]), 28, dtype=torch.float32)
    want = torch.cat([k[:20], 3 * k[20:22], k[30:36]])
    sc = cache.k_scale[:2].repeat_interleave(16, 0)[:28, :, None]
    assert ((kr - want).abs() <= 1.5 * sc).all() and torch.equal(kr, vr)


# ---------------------------------------------------------------- read

@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("P,D", [(16, 64), (32, 128), (64, 64), (128, 128)])
def test_read(fmt, dtype, P, D):
    lens, rows = [0, 3, P - 1, 2 * P + 5], [1, 0, P + 2, 3 * P]
    cache = make_cache(fmt, 16, 3, P, D, P)
    table = make_table(lens, rows, P, 16, 5)
    table[3, 3] = -1
    starts = np.concatenate([[0], np.cumsum(rows)])
    k, v = cache.read(ints(table), ints(lens), sum(rows), row_start=ints(starts), max_rows=max(rows), dtype=TD[dtype])
    h = host(cache)
    for got, name in ((k, "k"), (v, "v")):
        val = (ref.values(h[name], fmt).astype(np.float32) * h[name + "_scale"][:, :, None, None])
        for b in range(4):
            for r in range(starts[b], starts[b + 1]):
                p = lens[b] + r - starts[b]
                pg = table[b, p // P]
                want = val[pg, :, p % P] if pg >= 0 else np.zeros_like(val[0, :, 0])
                assert torch.equal(got[r].cpu(), torch.from_numpy(want).to(TD[dtype]))


# ---------------------------------------------------------------- streams, graphs, refusals

def test_streams_do_not_share_a_workspace():
    """Split calls in flight on two streams at once give the results of calls one after the other."""
    cache = make_cache("int8", 200, 2, 64, 64, 1)
    table, lens = ints(np.arange(200)[None]), ints([12000])
    q = [torch.randn(4, 8, 64, device="cuda").bfloat16() for _ in range(2)]
    want = [cache.attend(table, lens, x) for x in q]
    torch.cuda.synchronize()
    st = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(20):
        got = []
        for s, x in zip(st, q):
            with torch.cuda.stream(s):
                got.append(cache.attend(table, lens, x))
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_graph_capture():
    """append and attend in one graph: replays take the lengths and rows that lie there then."""
    cache = PagedCache.create(16, 2, 64, page_tokens=16)
    same = PagedCache.create(16, 2, 64, page_tokens=16)
    table, lens = ints(np.arange(16)[None]), ints([0])
    rotary = rotary_table(256, 64)
    x = torch.randn(1, 8, 64, device="cuda").bfloat16()

    def step(c, n):
        q = c.append(table, n, x[:, 4:6], x[:, 6:], q=x[:, :4], rotary=rotary)
        return c.attend(table, n, q)

    step(cache, lens)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(cache, lens)
        lens += 1
    lens.zero_()
    n = ints([0])
    for i in range(40):
        x.copy_(torch.randn(1, 8, 64, device="cuda").bfloat16())
        want = step(same, n)
        n += 1
        graph.replay()
        assert torch.equal(out, want), i


def test_zero_rows():
    cache = make_cache("int8", 4, 2, 16, 64, 1)
    table, lens = ints([[0, 1]]), ints([5])
    before = host(cache)
    e = torch.empty(0, 2, 64, device="cuda")
    cache.append(table, lens, e, e)
    assert cache.attend(table, lens, torch.empty(0, 4, 64, device="cuda")).shape == (0, 4, 64)
    assert cache.read(table, lens, 0)[0].shape == (0, 2, 64)
    assert (host(cache)["k"] == before["k"]).all()


def test_refusals():
    """Everything a call cannot take raises before a launch."""
    cache = make_cache("int8", 4, 2, 16, 64, 1)
    table, lens = ints([[0, 1]]), ints([5])
    q, k = torch.randn(2, 4, 64, device="cuda"), torch.randn(2, 2, 64, device="cuda")
    bad_attend = [dict(q=q.half()), dict(q=q[:, :3]), dict(q=q[:, :, :32]), dict(q=q.cpu()), dict(q=q[0]),
                  dict(q=q.transpose(0, 1).contiguous().transpose(0, 1)), dict(scale=0.0), dict(scale=float("nan")),
                  dict(softcap=-1.0), dict(window=-1), dict(slopes=torch.ones(3, device="cuda")),
                  dict(slopes=torch.ones(4)), dict(table=table.long()), dict(table=table[0]), dict(table=table.cpu()),
                  dict(lens=lens.long()), dict(lens=ints([1, 2])), dict(row_start=ints([0])),
                  dict(row_start=torch.tensor([0, 2], device="cuda")), dict(out=torch.empty(3, 4, 64, device="cuda")),
                  dict(out=q.bfloat16()), dict(max_rows=-1, row_start=ints([0, 2]))]
    for kw in bad_attend:
        a = dict(table=table, lens=lens, q=q)
        a.update(kw)
        with pytest.raises(ValueError):
            cache.attend(**a)
    odd = torch.randn(2, 600, device="cuda")
    bad_append = [dict(k=k.half()), dict(v=k.bfloat16()), dict(v=k[:1]), dict(k=odd[:, 1:129].view(2, 2, 64)),
                  dict(k=torch.randn(2, 133, device="cuda")[:, :128].view(2, 2, 64)), dict(q=q[:1]),
                  dict(q_out=q), dict(rotary=rotary_table(8, 64)[:, :, :1]), dict(rotary=rotary_table(8, 64).double()),
                  dict(rotary=rotary_table(8, 24)), dict(rotary=rotary_table(8, 128)), dict(lens=lens.cpu()),
                  dict(table=ints([[0], [1], [2]]), lens=ints([0, 0, 0]))]
    for kw in bad_append:
        a = dict(table=table, lens=lens, k=k, v=k)
        a.update(kw)
        with pytest.raises(ValueError):
            cache.append(**a)
    with pytest.raises(ValueError):
        cache.read(table, lens, 2, dtype=torch.float16)
    c = cache
    for args in ((c.k, c.v[:3], c.k_scale, c.v_scale), (c.k, c.v, c.k_scale[:3], c.v_scale),
                 (c.k.cpu(), c.v.cpu(), c.k_scale.cpu(), c.v_scale.cpu()), (c.k[:, :, :8], c.v[:, :, :8], c.k_scale, c.v_scale),
                 (c.k.float(), c.v.float(), c.k_scale, c.v_scale), (c.k, c.v, c.k_scale.double(), c.v_scale)):
        with pytest.raises(ValueError):
            PagedCache(*args)
    with pytest.raises(ValueError):
        PagedCache(c.k, c.v, c.k_scale, c.v_scale, fmt="int4")
