"""token_probs against its definition in 64 bits: sizes, cuts, ties, masked rows, strides, settings, streams, graphs."""
import numpy as np
import pytest
import torch

from sampling_ref import probs as ref

pytestmark = pytest.mark.gpu


def logits(n, V, seed, dtype=torch.float32, std=2.5):
    g = np.random.default_rng(seed)
    x = g.normal(0, std, (n, V))
    at = g.integers(0, V, (n, 8))
    np.put_along_axis(x, at, np.take_along_axis(x, at, 1) + g.uniform(2, 9, (n, 8)), 1)
    return torch.tensor(x, dtype=torch.float32).to(dtype)


def each(v, n):
    return v.tolist() if isinstance(v, torch.Tensor) else [v] * n


def check(x, T=1.0, k=0, p=1.0, out=None, flags=0, **kw):
    """One call on rows x (device), every entry against the definition."""
    from paper_2510_05421_gb300 import token_probs
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = token_probs(x, T, k, p, out=out, status=status, **kw)
    torch.cuda.synchronize()
    assert got.dtype == torch.float32 and got.shape == x.shape and (out is None or got is out)
    assert int(status) == flags
    host = got.cpu().double().numpy()
    for r, (t, kk, pp) in enumerate(zip(each(T, len(x)), each(k, len(x)), each(p, len(x)))):
        want, tol, border = ref(x[r].double().cpu().numpy(), np.float32(t), kk, float(np.float32(pp)))
        # a decision this near its border is not this test's: the inputs are chosen so that there is none
        assert border > 1e-10
        # tokens that stay are above 0, the others 0 (one below 2^-140 of the sum may be lost: f32 ends at 2^-149)
        assert (host[r] > 0)[want > 2.0 ** -140].all() and (host[r] == 0)[want == 0].all(), f"row {r}: tokens that stay"
        assert (np.abs(host[r] - want) <= tol).all(), (r, np.abs(host[r] - want).max())
    return got


SIZES = [(1, 1), (3, 2), (2, 31), (1, 33), (4, 1000), (2, 1024), (3, 4099), (2, 16384), (2, 16385), (3, 32000), (2, 50001),
         (1, 131072), (2, 200003), (1, 262144)]


@pytest.mark.parametrize("n,V", SIZES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_temperature(n, V, dtype):
    check(logits(n, V, V, dtype).cuda(), 0.8)


@pytest.mark.parametrize("n,V", SIZES)
@pytest.mark.parametrize("k,p", [(0, 0.9), (40, 1.0), (300, 0.7), (1, 0.5), (0, 0.0)])
def test_cuts(n, V, k, p):
    check(logits(n, V, 7 * V + n).cuda(), 0.9, k, p)


@pytest.mark.parametrize("std,T", [(0.01, 1.0), (30.0, 1.0), (2.0, 0.05), (2.0, 5.0), (1e-6, 1.0), (2.0, 1e-30), (2.0, 1e30)])
@pytest.mark.parametrize("k,p", [(0, 1.0), (0, 0.8), (500, 0.95)])
def test_flat_and_peaked_rows(std, T, k, p):
    check(logits(2, 5003, 11, std=std).cuda(), T, k, p)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [7, 2048, 20011, 140000])
@pytest.mark.parametrize("k,p", [(5, 1.0), (0, 0.3), (999, 0.301), (0, 1.0)])
def test_equal_logits_stay_in_order_of_their_index(V, k, p, dtype):
    x = torch.full((2, V), 1.5, dtype=dtype)
    x[1, ::3] = 2.0
    check(x.cuda(), 1.0, k, p)


@pytest.mark.parametrize("k,p", [(50, 1.0), (0, 0.9), (20, 0.6)])
def test_bf16_ties_at_the_cut(k, p):
    x = logits(8, 32000, 5, torch.bfloat16)
    top = x.float().sort(-1, descending=True).values
    assert p < 1 or bool((top[:, k - 1] == top[:, k]).any())
    check(x.cuda(), 0.7, k, p)


def test_zeros_of_either_sign_are_equal():
    x = torch.zeros(1, 300)
    x[0, ::2] = -0.0
    check(x.cuda(), 1.0, 7, 1.0)


@pytest.mark.parametrize("low", [-float("inf"), -3.0e38, float(torch.finfo(torch.bfloat16).min)])
@pytest.mark.parametrize("k,p", [(0, 1.0), (0, 0.9), (10, 1.0), (100, 0.99)])
def test_masked_tokens(low, k, p):
    """Grammar masks: most tokens at the lowest value; rows where one, three or none are left."""
    g = torch.Generator().manual_seed(2)
    x = logits(4, 3001, 3)
    x = torch.where(torch.rand(x.shape, generator=g) < 0.9, low, x)
    x[1] = low
    x[1, 1234] = -2.0
    x[2] = low
    x[2, [0, 17, 3000]] = 0.25
    x[3] = -float("inf")
    got = check(x.cuda(), 1.3, k, p)
    assert int(torch.count_nonzero(got[3])) == 0


def test_logits_that_are_no_numbers():
    x = logits(5, 2500, 4)
    x[0, 7] = float("nan")
    x[1] = float("nan")
    x[2, [3, 99]] = float("inf")
    for r in range(3):
        check(x[r:r + 1].cuda(), 0.9, 40, 0.9, flags=1)
    check(x.cuda(), 1.0, flags=1)
    check(x[3:].cuda(), 1.0)


def test_settings_of_each_row():
    n, V = 12, 9001
    x = logits(n, V, 6).cuda()
    T = torch.tensor([0, 1, .5, 0, 2, 1, 1, .7, 1e-3, 1, 1, 3], dtype=torch.float32).cuda()
    k = torch.tensor([0, 0, 5, 3, 0, 1, 9001, 99999, 0, 700, 2, 0], dtype=torch.int32).cuda()
    p = torch.tensor([.5, .9, 1, 1, .95, .5, 1, .8, .5, 2, 0, .999], dtype=torch.float32).cuda()
    check(x, T, k, p)
    check(x, T)
    check(x, 0.8, k)
    check(x, 0.8, 0, p)
    check(x.bfloat16(), T, 0, 0.9)


def test_greedy_is_the_first_of_the_largest():
    x = logits(6, 32000, 8)
    x[2, [5, 77]] = 50.0
    check(x.cuda(), 0.0)
    check(x.bfloat16().cuda(), 0.0, 3, 0.5)


def test_odd_settings_in_tensors():
    """Negative temperatures are greedy, a negative top_k cuts nothing; NaN is flagged."""
    x = logits(3, 1000, 9).cuda()
    f = lambda *v: torch.tensor(v, dtype=torch.float32).cuda()
    check(x, f(-1, 1, 1), torch.tensor([0, -5, 3], dtype=torch.int32).cuda(), f(1, 1, -2))
    from paper_2510_05421_gb300 import token_probs
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    nan = float("nan")
    got = token_probs(x, f(nan, 1, 1), 0, f(1, nan, 1), status=st)
    assert int(st) == 1 and torch.equal(got, token_probs(x, f(0, 1, 1), 0, f(1, 1, 1)))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pad,shift", [(1, 0), (64, 0), (7, 3), (0, 1), (5, 2)])
def test_strides(pad, shift, dtype):
    """Rows that lie apart and start anywhere; what lies between them is not written."""
    n, V = 5, 4001
    buf = torch.full((n * (V + pad) + 8,), 1e30, dtype=dtype, device="cuda")
    x = buf[shift:shift + n * (V + pad)].view(n, V + pad)[:, :V]
    x.copy_(logits(n, V, 10).to(dtype))
    out = torch.full((n, V + 2 * pad + 1), -7.0, device="cuda")
    check(x, 0.9, 100, 0.9, out=out[:, pad:pad + V])
    assert bool((out[:, :pad] == -7).all()) and bool((out[:, pad + V:] == -7).all())


def test_rows_past_32_bits_of_offset():
    V, ld = 1000, 1 << 30
    buf = torch.empty(2 * ld + V, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((3, V), (ld, 1))
    x.copy_(logits(3, V, 12).to(torch.bfloat16))
    check(x, 1.0, 20)
    del buf, x
    buf = torch.empty(2 * ld + V, device="cuda")
    check(logits(3, V, 13).cuda(), 1.0, out=buf.as_strided((3, V), (ld, 1)))


def test_many_rows_and_none():
    from paper_2510_05421_gb300 import token_probs
    x = logits(1, 1031, 14).cuda()
    one = token_probs(x, 0.8, 30, 0.9)
    many = token_probs(x.expand(700, -1).contiguous(), 0.8, 30, 0.9)
    assert torch.equal(many, one.expand(700, -1))                 # a row does not depend on how many there are
    assert token_probs(x[:0], 0.8).shape == (0, 1031)
    assert torch.equal(token_probs(x.expand(3, -1).contiguous()[:1], 0.8, 30, 0.9), one)


def test_same_bits_every_time():
    from paper_2510_05421_gb300 import token_probs
    x = logits(64, 32000, 15, torch.bfloat16).cuda()
    first = token_probs(x, 0.9, 0, 0.95)
    for _ in range(5):
        assert torch.equal(token_probs(x, 0.9, 0, 0.95), first)


def test_stream_and_graph():
    from paper_2510_05421_gb300 import token_probs
    x = logits(9, 7001, 16).cuda()
    want = token_probs(x, 0.9, 50, 0.9)
    side = torch.cuda.Stream()
    y = x.clone()                                   # in flight on the current stream
    got = token_probs(y, 0.9, 50, 0.9, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    T = torch.full((9,), 0.9, device="cuda")
    with torch.cuda.graph(graph):
        got = token_probs(y, T, 50, 0.9)
    y.copy_(logits(9, 7001, 17).cuda())
    T[4] = 0.0
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, token_probs(y, T, 50, 0.9))
    assert torch.count_nonzero(got[4]) == 1


@pytest.mark.parametrize("V", [500, 4099, 32000, 200003])
@pytest.mark.parametrize("kw", [dict(), dict(top_p=0.9), dict(top_k=30), dict(temperature=0.0)])
def test_in_place(V, kw):
    from paper_2510_05421_gb300 import token_probs
    x = logits(9, V, 20).cuda()
    want = token_probs(x, **kw)
    assert token_probs(x, out=x, **kw) is x
    assert torch.equal(x, want)


def test_refusals():
    from paper_2510_05421_gb300 import token_probs
    x = logits(3, 100, 18).cuda()
    f = torch.ones(3, device="cuda")
    for bad in (dict(temperature=-1.0), dict(temperature=float("nan")), dict(top_k=-1), dict(top_p=-0.1),
                dict(temperature=f[:2]), dict(temperature=f.double()), dict(top_k=f), dict(top_p=f.cpu()),
                dict(out=x.bfloat16()), dict(out=x[:2]), dict(status=f), dict(top_p=torch.ones(6, device="cuda")[::2])):
        with pytest.raises(ValueError):
            token_probs(x, **bad)
    for y in (x.half(), x[0], x.cpu(), x.t(), torch.empty(1, 262145, device="cuda"), torch.empty(2, 0, device="cuda")):
        with pytest.raises(ValueError):
            token_probs(y)


@pytest.mark.parametrize("p", [0.99, 0.9999, 0.9999999, 1 - 2.0 ** -24])
@pytest.mark.parametrize("T", [0.25, 1.0])
@pytest.mark.parametrize("V", [3000, 100003])
def test_cuts_deep_in_the_tail(V, T, p):
    """top_p just below 1: the last kept token's w is down to 2^-40 of the largest, or below what a mass resolves."""
    from paper_2510_05421_gb300 import token_probs
    x = logits(2, V, 19)
    got = token_probs(x.cuda(), T, 0, p).cpu().double().numpy()
    p = float(np.float32(p))
    for r in range(2):
        v = x[r].double().numpy()
        w = np.exp((v - v.max()) / np.float32(T))
        order = np.argsort(-v, kind="stable")
        kept = int((got[r] > 0).sum())
        assert (got[r][order[:kept]] > 0).all()                     # a prefix of the order
        # its end is where the sum reaches p of the whole, within what the masses' rounding may move: each is off by
        # less than 2^-44 and by 2^-33 of itself, and counts once: before p of the whole or behind it
        before, all_of_it = w[order].cumsum() - w[order], w.sum()
        slack = V * 2.0 ** -44 + all_of_it * 2.0 ** -33
        assert before[kept - 1] < p * all_of_it + slack and (kept == V or before[kept] >= p * all_of_it - slack)
        want = np.where(np.isin(np.arange(V), order[:kept]), w, 0) / w[order[:kept]].sum()
        t = np.abs((v - v.max()) / np.float32(T))
        assert (np.abs(got[r] - want) <= want * (t * 3 * 2.0 ** -24 + 2.0 ** -21) + 2.0 ** -140).all()


@pytest.mark.parametrize("V", [3001, 32000, 128001])
@pytest.mark.parametrize("k", [1, 50, 400, 512, 513, 1024, 1025, 2999])
def test_top_k_where_the_likeliest_lie_together(V, k):
    """The largest logits one after another (one CTA, a few threads have them all), or spread by a stride of the threads."""
    n = min(V, 1500)
    x = logits(4, V, 21)
    g = torch.Generator().manual_seed(1)
    top = 12 + 3 * torch.rand(n, generator=g)
    x[0, :n] = top
    x[1, V - n:] = top
    at = torch.arange(0, V, 512)[:n]
    x[2, at] = top[:len(at)]
    x[3, :n] = top.bfloat16().float()                           # with ties
    check(x.cuda(), 1.0, k)
    check(x.cuda(), 1.0, k, 0.9)


@pytest.mark.parametrize("V", [32000, 128001])
@pytest.mark.parametrize("p", [0.1137, 0.5377, 0.9861])
@pytest.mark.parametrize("how", ["wide", "dense", "sorted", "lumps", "two"])
def test_many_tokens_where_the_cut_is(V, p, how):
    """More tokens lie together at top_p's cut than are sorted out at once: spread evenly, in order, in lumps."""
    g = torch.Generator().manual_seed(int(p * 1e4) + V)
    if how == "wide":                                           # logits as they are, the cut far below the largest
        x, T = logits(6, V, 23, std=2.0) + torch.tensor([[0.0], [1.0], [2.0], [3.0], [4.0], [5.0]]) * 0.01, 0.78
        x[:, 7] = 17.0
    elif how == "dense":
        x, T = 5 + 1e-3 * torch.rand(3, V, generator=g), 1.0
    elif how == "sorted":
        x, T = (5 + 1e-2 * torch.rand(3, V, generator=g)).sort(-1)[0], 1.0
    elif how == "lumps":                                        # most of them equal, the others on one side or both
        x, T = 5 + 1e-2 * torch.rand(3, V, generator=g), 1.0
        lump = torch.rand(3, V, generator=g) < torch.tensor([[0.5], [0.9], [0.99]])
        x[lump] = torch.tensor([[5.001], [5.009], [5.005]]).expand(3, V)[lump]
    else:                                                       # two values, next to each other
        x, T = torch.where(torch.rand(3, V, generator=g) < 0.5, 5.0, 5.0 + 2.0 ** -21), 1.0
    check(x.cuda(), T, 0, p)


def test_rows_beside_each_other_and_over_each_other():
    from paper_2510_05421_gb300 import DVIError, token_probs
    V = 1000
    buf = torch.zeros(5, 2 * V + 8, device="cuda")
    x = logits(5, V, 24).cuda()
    for cuts in (dict(), dict(top_k=20, top_p=0.9)):
        want = token_probs(x, **cuts)
        buf[:, 4:V + 4] = x
        assert torch.equal(token_probs(buf[:, 4:V + 4], out=buf[:, V + 4:2 * V + 4], **cuts), want)
        assert torch.equal(buf[:, 4:V + 4], x)
        for out in (buf[:, 5:V + 5], buf[:, :V], buf[:, V + 3:2 * V + 3]):
            with pytest.raises(DVIError):
                token_probs(buf[:, 4:V + 4], out=out, **cuts)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1, 6, 1019, 4097, 16381, 65531, 131069, 262137, 262144])
@pytest.mark.parametrize("shift,out_shift", [(0, 0), (1, 1), (3, 7), (6, 2), (5, 0), (7, 3)])
def test_rows_that_begin_anywhere(V, shift, out_shift, dtype):
    """Between numbers that would show if they were read, and that show if they are written; rows of odd lengths one after
    another, so that each begins elsewhere in its 16 bytes."""
    n = 3
    buf = torch.full((n * V + 16,), float("nan"), dtype=dtype, device="cuda")
    x = buf[shift:shift + n * V].view(n, V)
    x.copy_(logits(n, V, 25).to(dtype))
    for kw in (dict(), dict(T=0.0), dict(k=60), dict(p=0.9)):
        room = torch.full((n * V + 16,), -7.0, device="cuda")
        check(x, out=room[out_shift:out_shift + n * V].view(n, V), **kw)
        assert bool((room[:out_shift] == -7).all()) and bool((room[out_shift + n * V:] == -7).all())


@pytest.mark.parametrize("V", [1021, 50257, 100003])
@pytest.mark.parametrize("kw", [dict(), dict(top_p=0.9), dict(top_k=30), dict(temperature=0.0)])
def test_odd_rows_in_place(V, kw):
    from paper_2510_05421_gb300 import token_probs
    x = logits(5, V, 26).cuda()
    want = token_probs(x, **kw)
    assert token_probs(x, out=x, **kw) is x
    assert torch.equal(x, want)


@pytest.mark.parametrize("kw", [dict(T=0.7), dict(T=0.7, p=0.9), dict(T=0.7, k=40, p=0.8), dict(T=1e-4, p=0.5),
                                dict(T=30.0, p=0.999), dict(T=1e-5, k=3, p=0.9)])
@pytest.mark.parametrize("shift", [0.0, 40.0, -500.0, 3e4, -3e4])
def test_logits_far_from_zero(shift, kw):
    """Rows that lie far up or down: their distance from the largest counts, not where it is."""
    x = logits(3, 20000, 27) + shift
    check(x.cuda(), **kw)


@pytest.mark.parametrize("V", [1, 2, 32, 33, 127, 600, 1024, 1025, 2047, 2048, 2049])
@pytest.mark.parametrize("how", ["normal", "ties", "masked", "infinite", "equal", "lump", "apart", "near"])
def test_short_rows(V, how):
    g = torch.Generator().manual_seed(V)
    x = logits(6, V, 28)
    if how == "ties":
        x = x.bfloat16().float()
    elif how in ("masked", "infinite"):                         # a few are left, one, none
        low = -3.0e38 if how == "masked" else -float("inf")
        x[torch.rand(6, V, generator=g) < 0.95] = low
        x[4], x[5] = low, low
        x[4, V // 2] = 1.0
    elif how == "equal":
        x[:] = torch.tensor([-7.0, 0.0, 1e-40, 3e38, -3e38, 0.125])[:, None]
    elif how == "lump":                                         # many equal ones at the top, in the middle, at the end
        x[:, ::3] = torch.tensor([20.0, 2.0, 0.0, -3.0, -20.0, -1e30])[:, None]
    elif how == "apart":                                        # by orders of magnitude, on both sides of 0
        x = torch.exp(60 * (torch.rand(6, V, generator=g) - 0.7)) * torch.where(torch.rand(6, V, generator=g) < 0.5, -1, 1)
    elif how == "near":                                         # neighbours, as far as f32 tells them apart
        x = 1.0 + torch.randint(0, V, (6, V), generator=g) * 2.0 ** -23
    for k, p in ((1, 1.0), (31, 1.0), (40, 0.9), (500, 1.0), (0, 0.3717), (0, 0.9137), (1000, 0.5113), (V - 1, 0.0)):
        check(x.cuda(), 0.9, k, p)
