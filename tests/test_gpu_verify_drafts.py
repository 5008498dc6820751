"""verify_drafts against its definition in 64 bits: ragged batches, rejected and bonus rows, odd probabilities, and the
distribution of what it commits."""
import numpy as np
import pytest
import torch

from sampling_ref import verify as ref

pytestmark = pytest.mark.gpu


def case(counts, V, seed, bonus, greedy=False, noise=0.7, cut=1e-4):
    g = np.random.default_rng(seed)
    n, B = sum(counts), len(counts)
    x = g.normal(0, 2.0, (n + B * bonus, V))
    x[np.arange(len(x)), g.integers(0, V, len(x))] += 6
    p = np.exp(x - x.max(-1, keepdims=True))
    p[p < cut * p.max(-1, keepdims=True)] = 0
    p /= p.sum(-1, keepdims=True)
    rows = [r + b * bonus for b, (a, c) in enumerate(zip(np.cumsum([0, *counts]), counts)) for r in range(a, a + c)]
    z = x[rows] + g.normal(0, noise, (n, V))
    q = np.exp(z - z.max(-1, keepdims=True)) if n else z
    q /= q.sum(-1, keepdims=True)
    ids = z.argmax(-1) if greedy else np.array([g.choice(V, p=r) for r in q], dtype=np.int64)
    return (p.astype(np.float32), ids.astype(np.int32).reshape(-1), g.random(n, dtype=np.float32),
            g.random(B, dtype=np.float32), None if greedy else q.astype(np.float32))


def run(p, ids, ua, ut, q, counts, bonus, ragged=None, most=None, flags=0, **kw):
    from paper_2510_05421_gb300 import verify_drafts
    ragged = len(set(counts)) > 1 if ragged is None else ragged
    d = lambda v: torch.from_numpy(np.ascontiguousarray(v)).cuda()
    start = d(np.cumsum([0, *counts]).astype(np.int32)) if ragged else None
    most = max([*counts, 0]) if most is None else most
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = verify_drafts(d(p) if isinstance(p, np.ndarray) else p, d(ids), d(ua), d(ut),
                        draft=d(q) if isinstance(q, np.ndarray) else q, draft_start=start, max_drafts=most, bonus=bonus,
                        status=status, **kw)
    torch.cuda.synchronize()
    assert int(status) == flags
    return [t.cpu().numpy() for t in got]


def check(p, ids, ua, ut, q, counts, bonus, **kw):
    got = run(p, ids, ua, ut, q, counts, bonus, **kw)
    want = ref(p, ids, ua, ut, q, counts, int(bonus), kw.get("most"))
    for a, b in zip(got, want):
        np.testing.assert_array_equal(a, b)
    return got


@pytest.mark.parametrize("V", [1, 2, 33, 1000, 1024, 4099, 32000, 50001, 131073, 262144])
@pytest.mark.parametrize("counts", [[1], [5], [0], [3, 0, 7, 1], [4] * 6])
@pytest.mark.parametrize("bonus", [True, False])
def test_sizes(V, counts, bonus):
    for greedy in (False, True):
        c = case(counts, V, V + len(counts), int(bonus), greedy)
        check(*c, counts, bonus)


@pytest.mark.parametrize("B", [1, 8, 64, 200])
@pytest.mark.parametrize("V", [999, 32000])
def test_batches(B, V):
    counts = [(7 * b) % 9 for b in range(B)]
    got = check(*case(counts, V, B, 1), counts, True)
    if B >= 64:
        m = got[2]
        assert (m == np.array(counts)).any() and (m < np.array(counts)).any()


@pytest.mark.parametrize("counts", [[40], [32], [33, 64, 100]])
def test_long_blocks(counts):
    """More drafts than a warp has lanes; rows equal to the drafter's, so that all are accepted up to a planted one."""
    p, ids, ua, ut, q = case(counts, 500, 3, 1, noise=0.0, cut=0.0)
    for last in (31, 32, 39, 99):
        u = ua * 0.9
        if last < len(u):
            u[last] = 1.0
            p2 = p.copy()
            q2 = q.copy()
            row = last + sum(last >= s for s in np.cumsum(counts)[:-1])
            p2[row, ids[last]] *= 0.5
            check(p2, ids, u, ut, q2, counts, True)
    check(p, ids, ua * 0.9, ut, q, counts, True)


def test_first_and_last_tokens_of_a_row():
    """Uniform numbers at their ends, and rows whose only numbers are at the row's ends."""
    V = 5000
    p = np.zeros((4, V), np.float32)
    p[0, 0] = p[1, V - 1] = 1.0
    p[2, [0, V - 1]] = 0.5
    p[3] = 1.0 / V
    none = np.zeros(0, np.int32), np.zeros(0, np.float32)
    for u in (0.0, 0.25, 0.5, 0.75, 1.0 - 2.0 ** -24):
        check(p, *none, np.full(4, u, np.float32), None, [0] * 4, True)
    # out of [0, 1): as the nearest number in it
    lo = run(p, *none, np.array([-1, -1, -1, -1], np.float32), None, [0] * 4, True)[0][:, 0]
    hi = run(p, *none, np.array([2, 2, 2, 1], np.float32), None, [0] * 4, True)[0][:, 0]
    nan = run(p, *none, np.full(4, np.nan, np.float32), None, [0] * 4, True)[0][:, 0]
    assert lo.tolist() == [0, V - 1, 0, 0] and hi.tolist() == [0, V - 1, V - 1, V - 1] and nan.tolist() == lo.tolist()


def test_rows_that_are_equal_or_empty():
    V = 700
    p, ids, ua, ut, q = case([2, 2, 2], V, 5, 1)
    ua[:] = 1.0                                     # p = q is accepted for u < 1 alone
    p[0] = q[0]                                     # rejected, and nothing is left: a token of p
    p[3] = 0.0                                      # an empty row: no token
    p[6] = q[4]
    check(p, ids, ua, ut, q, [2, 2, 2], True, flags=1)


def test_numbers_that_are_no_probabilities():
    V = 1500
    p, ids, ua, ut, q = case([3, 3, 3, 3], V, 6, 1)
    p *= 3.0                                        # they need not sum to 1
    check(p, ids, ua, ut, q, [3] * 4, True)
    ua[:] = 0.999999
    p[0, ::2] = np.nan
    p[4, 1::2] = np.inf
    q[6, ::3] = np.nan
    p[12] = np.nan
    p[1, ::5] = -1.0
    check(p, ids, ua, ut, q, [3] * 4, True, flags=1)


@pytest.mark.parametrize("greedy", [False, True])
def test_ids_outside_the_vocabulary(greedy):
    V = 800
    c = list(case([2, 2, 2], V, 7, 1, greedy))
    c[2] *= 0.0                                     # everything else is accepted where p > 0
    c[0] = np.maximum(c[0], 1e-6)
    c[1][[0, 3]] = V, -1
    got = check(*c, [2, 2, 2], True, flags=8)
    assert got[2].tolist() == [0, 1, 2]


def test_max_drafts_below_the_longest():
    """Drafts past max_drafts are not looked at; the bonus row is then the next draft's."""
    counts = [5, 2, 7, 0]
    p, ids, ua, ut, q = case(counts, 600, 8, 1)
    for most in (0, 1, 3, 7, 12):
        check(p, ids, ua * 0.2, ut, q, counts, True, most=most)


def test_starts_out_of_order_stay_inside():
    """Row starts that fall or point past the drafts: nothing outside the arrays is read, the others are right."""
    from paper_2510_05421_gb300 import verify_drafts
    p, ids, ua, ut, q = (torch.from_numpy(t).cuda() for t in case([2, 2, 2], 300, 9, 1))
    start = torch.tensor([0, 2, -5, 1 << 30], dtype=torch.int32).cuda()
    got = verify_drafts(p, ids, ua, ut, draft=q, draft_start=start, max_drafts=2)
    want = verify_drafts(p, ids, ua, ut, draft=q, max_drafts=2)
    torch.cuda.synchronize()
    assert torch.equal(got[0][0], want[0][0]) and int(got[2][1]) == 0


@pytest.mark.parametrize("start,flag", [([0, 2, 4, 6], 0), ([0, 2, 6, 6], 0), ([1, 2, 3, 5], 0), ([0, 4, 2, 6], 8),
                                        ([0, 2, 4, 7], 8), ([-1, 2, 4, 6], 8), ([0, 2, 4, -1], 8)])
def test_starts_out_of_order_are_flagged(start, flag):
    from paper_2510_05421_gb300 import verify_drafts
    p, ids, ua, ut, q = (torch.from_numpy(t).cuda() for t in case([2, 2, 2], 300, 9, 1))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    verify_drafts(p, ids, ua, ut, draft=q, draft_start=torch.tensor(start, dtype=torch.int32).cuda(), max_drafts=6,
                  status=status)
    assert int(status) == flag


def test_committed_tokens_are_distributed_as_the_targets():
    """One draft, a grid of both uniform numbers: the committed first token has the target's probabilities.  A cell of
    the grid is 2^-8 wide; acceptance and each of the V ranges of the token can be off by one cell."""
    V, N = 6, 256
    g = np.random.default_rng(0)
    p, q = g.dirichlet(np.ones(V)), g.dirichlet(np.ones(V))
    p[2] = 0
    p /= p.sum()
    u = (np.arange(N) + 0.5) / N
    ua, ut = (v.reshape(-1).astype(np.float32) for v in np.meshgrid(u, u))
    freq = np.zeros(V)
    for x in range(V):
        ids = np.full(N * N, x, np.int32)
        got = run(np.tile(p.astype(np.float32), (N * N, 1)), ids, ua, ut, np.tile(q.astype(np.float32), (N * N, 1)),
                  [1] * (N * N), False)
        freq += q[x] * np.bincount(got[0][:, 0], minlength=V) / N ** 2
        assert (got[1] == 1).all()
    assert np.abs(freq - p).max() <= 2 / N and freq[2] == 0


def test_sampled_tokens_have_the_probabilities():
    """No drafts: N equally spaced uniform numbers pick each token as often as its probability says, within one."""
    V, N = 40, 4096
    p = np.random.default_rng(1).dirichlet(np.ones(V) * 0.3).astype(np.float32)
    ut = ((np.arange(N) + 0.5) / N).astype(np.float32)
    got = run(np.tile(p, (N, 1)), np.zeros(0, np.int32), np.zeros(0, np.float32), ut, None, [0] * N, True)
    assert np.abs(np.bincount(got[0][:, 0], minlength=V) - p / p.sum(dtype=np.float64) * N).max() <= 1.01


def test_strides_and_offsets():
    counts = [3, 1, 4]
    p, ids, ua, ut, q = case(counts, 1001, 10, 1)
    wide = lambda v: torch.nn.functional.pad(torch.from_numpy(v), (1, 5), value=float("nan")).cuda()[:, 1:-5]
    got = run(wide(p), ids, ua, ut, wide(q), counts, True)
    for a, b in zip(got, ref(p, ids, ua, ut, q, counts, 1)):
        np.testing.assert_array_equal(a, b)


def test_rows_past_32_bits_of_offset():
    counts, V, ld = [1, 1], 500, 1 << 30
    p, ids, ua, ut, q = case(counts, V, 11, 1)
    buf = torch.empty(3 * ld + V, device="cuda")
    far = buf.as_strided((4, V), (ld, 1))
    far.copy_(torch.from_numpy(p))
    for u in (0.0, 1.0):
        got = run(far, ids, ua * 0 + u, ut, q, counts, True)
        for a, b in zip(got, ref(p, ids, ua * 0 + u, ut, q, counts, 1)):
            np.testing.assert_array_equal(a, b)


def test_stream_and_graph():
    from paper_2510_05421_gb300 import verify_drafts
    counts = [4] * 5
    a = [torch.from_numpy(t).cuda() for t in case(counts, 3001, 12, 1)]
    b = [torch.from_numpy(t).cuda() for t in case(counts, 3001, 13, 1)]
    call = lambda p, ids, ua, ut, q, **kw: verify_drafts(p, ids, ua, ut, draft=q, **kw)
    want_a, want_b = call(*a), call(*b)
    side = torch.cuda.Stream()
    got = call(*a, stream=side)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want_a))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call(*a)
    for x, y in zip(a, b):
        x.copy_(y)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want_b))


def test_nothing_to_do():
    from paper_2510_05421_gb300 import verify_drafts
    z = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype, device="cuda")
    ids, nc, na = verify_drafts(z(0, 9), z(0, dtype=torch.int32), z(0), z(0))
    assert ids.shape == (0, 1) and nc.numel() == na.numel() == 0
    ids, nc, na = verify_drafts(z(0, 9), z(0, dtype=torch.int32), z(0), z(3), bonus=False)
    assert ids.shape == (3, 0) and nc.tolist() == na.tolist() == [0, 0, 0]


def test_refusals():
    from paper_2510_05421_gb300 import verify_drafts
    p, ids, ua, ut, q = (torch.from_numpy(t).cuda() for t in case([2, 2], 50, 14, 1))
    ok = dict(target=p, draft_ids=ids, u_accept=ua, u_token=ut, draft=q)
    verify_drafts(**ok)
    s = torch.tensor([0, 2, 4], dtype=torch.int32).cuda()
    for bad in (dict(target=p[:5]), dict(target=p.bfloat16()), dict(target=p.cpu()), dict(target=p.t()), dict(draft_ids=ids.long()),
                dict(draft_ids=ids[:3]), dict(u_accept=ua[:3]), dict(u_accept=ua.double()), dict(u_token=ut.cpu()),
                dict(draft=q[:3]), dict(draft=q[:, :49]), dict(draft=q.half()), dict(draft_start=s[:2]),
                dict(draft_start=s.long()), dict(max_drafts=1), dict(max_drafts=-1), dict(bonus=False),
                dict(status=ut), dict(draft_start=s, max_drafts=(1 << 20) + 1)):
        with pytest.raises(ValueError):
            verify_drafts(**{**ok, **bad})
