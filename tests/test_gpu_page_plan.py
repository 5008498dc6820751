"""PagePool against lists: growth, rollback, ending sequences, pools that run short, rows and slots, graphs."""
import numpy as np
import pytest
import torch

from sampling_ref import Pool

pytestmark = pytest.mark.gpu


def dev(v):
    return torch.tensor(v, dtype=torch.int32).cuda()


def same(pool, ref):
    torch.cuda.synchronize()
    assert pool.n_free.item() == len(ref.stack)
    assert pool.stack[:len(ref.stack)].tolist() == ref.stack
    assert pool.held.tolist() == [len(t) for t in ref.tables]
    np.testing.assert_array_equal(pool.table.cpu().numpy(), ref.table())


def step(pool, ref, lens, rows, n_rows=None):
    total = sum(max(t, 0) for t in rows)
    n = total if n_rows is None else n_rows
    start, slots, positions, full = ref.plan(lens, rows)
    got = pool.plan(dev(lens), dev(rows), n_rows=n)
    same(pool, ref)
    assert got.row_start.tolist() == start
    want = (slots + [-1] * n)[:n], (positions + [-1] * n)[:n]
    assert got.slots.tolist() == want[0] and got.positions.tolist() == want[1]
    assert pool.status() == (["KV_FULL"] if full or total > n else [])


@pytest.mark.parametrize("B,P,max_pages", [(1, 16, 5), (7, 16, 40), (33, 64, 9), (100, 32, 20), (1024, 128, 6)])
def test_sequences_come_grow_roll_back_and_end(B, P, max_pages):
    from paper_2510_05421_gb300 import PagePool
    g = np.random.default_rng(B)
    n_pages = B * max_pages                          # enough for all
    pool, ref = PagePool.create(n_pages, B, max_pages, P), Pool(n_pages, B, max_pages, P)
    lens = np.zeros(B, np.int64)
    for t in range(12):
        room = max_pages * P - lens
        rows = np.minimum(g.integers(0, 3 * P if t % 3 == 0 else 9, B), room) * (g.random(B) < 0.8)
        step(pool, ref, lens.tolist(), rows.tolist(), n_rows=None if t % 2 else int(rows.sum()) + 5)
        lens = lens + (rows * g.random(B)).astype(np.int64)
        lens[g.random(B) < 0.15] = 0
        pool.trim(dev(lens.tolist()))
        ref.plan(lens, [0] * B)
        same(pool, ref)
    pool.trim(dev([0] * B))
    ref.plan([0] * B, [0] * B)
    same(pool, ref)
    assert sorted(pool.stack.tolist()) == list(range(n_pages)) and pool.n_free.item() == n_pages


@pytest.mark.parametrize("B,n_pages", [(1, 3), (6, 10), (64, 70), (500, 900)])
def test_pools_that_run_short(B, n_pages):
    """What does not fit is passed over, the slots behind it get theirs."""
    from paper_2510_05421_gb300 import PagePool
    g, P, max_pages = np.random.default_rng(n_pages), 16, 8
    pool, ref = PagePool.create(n_pages, B, max_pages, P), Pool(n_pages, B, max_pages, P)
    short = 0
    for t in range(10):
        lens, rows = g.integers(0, max_pages * P // 2, B), g.integers(0, max_pages * P, B)
        if t == 4:
            rows = rows * 3                          # more than a table holds, too
        step(pool, ref, lens.tolist(), rows.tolist())
        short += len(ref.stack) < B
    assert short


def test_pages_given_back_are_taken_in_the_same_call():
    from paper_2510_05421_gb300 import PagePool
    pool, ref = PagePool.create(10, 3, 10, 16), Pool(10, 3, 10, 16)
    step(pool, ref, [0, 0, 0], [16 * 6, 16 * 3, 0])
    step(pool, ref, [0, 48, 0], [0, 16, 16 * 6])     # slot 0 ends, slot 2 takes its pages
    step(pool, ref, [0, 0, 0], [0, 0, 160])


def test_a_number_of_rows_for_all():
    from paper_2510_05421_gb300 import PagePool
    pool, ref = PagePool.create(64, 5, 8, 16), Pool(64, 5, 8, 16)
    lens = [0, 3, 15, 16, 17]
    ref.plan(lens, [0] * 5)
    pool.trim(dev(lens))
    got = pool.plan(dev(lens), 6, n_rows=30)
    start, slots, positions, _ = ref.plan(lens, [6] * 5)
    same(pool, ref)
    assert got.row_start.tolist() == start and got.slots.tolist() == slots and got.positions.tolist() == positions
    got = pool.plan(dev(lens), 6)
    assert got.slots is None and got.positions is None and got.row_start.tolist() == start


def test_odd_lengths():
    """Negative counts are 0; lengths and rows near 2^31 are passed over, and the sums do not wrap."""
    from paper_2510_05421_gb300 import PagePool
    big = 2 ** 31 - 1
    pool, ref = PagePool.create(20, 4, 5, 16), Pool(20, 4, 5, 16)
    step(pool, ref, [-5, 10, -1, 0], [3, -7, -2, 20])
    got = pool.plan(dev([big, 10, big, 0]), dev([big, 0, 1, big]), n_rows=4)
    torch.cuda.synchronize()
    assert got.row_start.tolist() == [0, big, big, big, big]
    assert got.slots.tolist() == [-1] * 4 and got.positions.tolist() == [big] * 4
    assert pool.status() == ["KV_FULL"]
    assert pool.held.tolist() == [1, 1, 0, 2]


def test_large_rows():
    """A long prompt in one slot among empty ones; slots past 32 bits."""
    from paper_2510_05421_gb300 import PagePool
    n = 70001
    pool, ref = PagePool.create(5000, 3, 4500, 16), Pool(5000, 3, 4500, 16)
    step(pool, ref, [0, 0, 0], [0, n, 0])
    far = PagePool.create(1 << 25, 2, 3, 128)        # the first pages come off the end
    far.stack.copy_(torch.arange(1 << 25, dtype=torch.int32))
    got = far.plan(dev([0, 100]), 200, n_rows=400)
    assert got.slots[0].item() == ((1 << 25) - 1) * 128 and got.slots[-1].item() > 2 ** 31


def test_a_pool_out_of_order_is_not_written_past():
    """Counts and pages out of their range: flagged, and the memory around the arrays stays."""
    from paper_2510_05421_gb300 import PagePool
    buf = torch.full((6, 64), 77, dtype=torch.int32, device="cuda")
    stack, n_free, held = buf[0, 8:16], buf[1, 8:9], buf[2, 8:11]
    table = buf[3, 8:20].view(3, 4)
    for n, h, t in ((50, [0, 0, 0], -1), (-3, [4, 4, 4], 3), (8, [9, -2, 4], 900), (8, [4, 4, 4], -1)):
        stack.copy_(torch.arange(8) * (100 if t == 900 else 1) - (5 if n == 50 else 0))
        n_free.fill_(n)
        held.copy_(dev(h))
        table.fill_(t)
        pool = PagePool(stack, n_free, table, held, 16)
        pool.plan(dev([0, 0, 0]), dev([16, 0, 40]), n_rows=56)
        pool.trim(dev([0, 0, 0]))
        pool.plan(dev([64, 64, 64]), 0)
        assert pool.status() == ["KV_FULL"]
        assert 0 <= n_free.item() <= 8 and bool(((held >= 0) & (held <= 4)).all())
        inside = torch.zeros_like(buf, dtype=torch.bool)
        inside[0, 8:16] = inside[1, 8:9] = inside[2, 8:11] = inside[3, 8:20] = True
        assert bool((buf[~inside] == 77).all())


def test_stream_and_graph():
    from paper_2510_05421_gb300 import PagePool
    pool, ref = PagePool.create(200, 6, 20, 16), Pool(200, 6, 20, 16)
    lens, rows = dev([0] * 6), dev([30, 5, 0, 64, 1, 16])
    side = torch.cuda.Stream()
    got = pool.plan(lens, rows, n_rows=116, stream=side)
    side.synchronize()
    start, slots, positions, _ = ref.plan([0] * 6, rows.tolist())
    same(pool, ref)
    assert got.slots.tolist() == slots
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = pool.plan(lens, rows, n_rows=40)
        pool.trim(lens)
    for t in range(4):
        new = [(b * 7 + 11 * t) % 90 for b in range(6)], [(3 * b + t) % 7 for b in range(6)]
        lens.copy_(dev(new[0]))
        rows.copy_(dev(new[1]))
        graph.replay()
        start, slots, positions, _ = ref.plan(*new)
        ref.plan(new[0], [0] * 6)
        same(pool, ref)
        assert got.row_start.tolist() == start and got.slots.tolist() == (slots + [-1] * 40)[:40]


def test_refusals():
    from paper_2510_05421_gb300 import PagePool
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    good = dict(stack=i(8), n_free=i(1), table=i(3, 4), held=i(3))
    PagePool(**good)
    for bad in (dict(stack=i(8).long()), dict(stack=i(8).cpu()), dict(n_free=i(2)), dict(table=i(12)), dict(held=i(4)),
                dict(table=i(4, 3).t()), dict(page_tokens=24), dict(stack=i(0)), dict(table=i(1025, 2), held=i(1025))):
        with pytest.raises(ValueError):
            PagePool(**{**good, **bad})
    pool = PagePool(**good)
    for args in ((i(4),), (i(3).long(),), (i(3).cpu(),), (i(3), -1), (i(3), i(2)), (i(3), i(3).float()),
                 (i(3), 0, -1), (i(3), 0, (1 << 30) + 1)):
        with pytest.raises(ValueError):
            pool.plan(*args)
    with pytest.raises(ValueError):
        pool.trim(i(2))
