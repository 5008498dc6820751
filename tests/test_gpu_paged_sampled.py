"""Page plans, the paged cache, token probabilities and verification together: a serving loop against its parts'
definitions, and PagedDecoder sampling over pages that the GPU hands out."""
import numpy as np
import pytest
import torch

import sampling_ref as ref
from gpu_helpers import teacher_forced_logits
from oracle import OracleModel
from paper_2510_05421_gb300 import DeviceWeights
from paper_2510_05421_gb300.paged_decode import PagedDecoder, Sampling, main
from workloads import make_prompts, make_weights, workload

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,V,K", [(1, 50, 3), (7, 3001, 4)])
def test_serving_steps(B, V, K):
    """Steps of sequences that come, draft, commit, roll back and end; the cache's rows lie in the plan's slots."""
    from paper_2510_05421_gb300 import PagedCache, PagePool, token_probs, verify_drafts
    g = np.random.default_rng(V)
    P, H, D, max_pages = 16, 2, 64, 12
    n_pages = B * max_pages
    cache = PagedCache.create(n_pages, H, D, P)
    pool, lists = PagePool.create(n_pages, B, max_pages, P), ref.Pool(n_pages, B, max_pages, P)
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    T, top_k, top_p = 0.9, 40, 0.95
    for t in range(8):
        prompts = t % 4 == 0
        counts = [int(n) for n in (g.integers(1, 30, B) if prompts else np.full(B, K + 1))]
        n = sum(counts)
        rows = torch.tensor(counts, dtype=torch.int32).cuda()
        plan = pool.plan(lens, rows, n_rows=n)
        start, slots, positions, full = lists.plan(lens.tolist(), counts)
        assert not full and plan.slots.tolist() == slots and plan.row_start.tolist() == start
        k, v = (torch.randn(n, H, D, device="cuda").bfloat16() for _ in range(2))
        cache.append(pool.table, lens, k, v, row_start=plan.row_start, max_rows=max(counts))
        kr, vr = cache.read(pool.table, lens, n, row_start=plan.row_start, max_rows=max(counts), dtype=torch.float32)
        page, off = plan.slots // P, plan.slots % P
        assert torch.equal(cache.k[page, :, off].float() * cache.k_scale[page][..., None], kr)
        assert torch.equal(cache.v[page, :, off].float() * cache.v_scale[page][..., None], vr)
        assert (kr - k.float()).abs().max() < 0.05      # (half a code of a scale of at most 5 / 127, and bf16)
        if prompts:
            lens = lens + rows
            continue
        z = torch.from_numpy(g.normal(0, 2, (B * (K + 1), V)).astype(np.float32)).cuda()
        d = z.view(B, K + 1, V)[:, :K].reshape(B * K, V) + torch.from_numpy(g.normal(0, .5, (B * K, V)).astype(np.float32)).cuda()
        q, p = token_probs(d, T, top_k, top_p), token_probs(z, T, top_k, top_p)
        ids = verify_drafts(q, rows.new_empty(0), q.new_empty(0), torch.from_numpy(g.random(B * K, dtype=np.float32)).cuda())[0][:, 0]
        ua, ut = (torch.from_numpy(g.random(m, dtype=np.float32)).cuda() for m in (B * K, B))
        out, n_committed, n_accepted = verify_drafts(p, ids, ua, ut, draft=q, max_drafts=K)
        want = ref.verify(p.cpu().numpy(), ids.cpu().numpy(), ua.cpu().numpy(), ut.cpu().numpy(), q.cpu().numpy(), [K] * B, 1)
        for a, b in zip((out, n_committed, n_accepted), want):
            np.testing.assert_array_equal(a.cpu().numpy(), b)
        lens = lens + n_committed
        if t == 5:
            lens = torch.where(torch.arange(B, device="cuda") % 2 == 0, 0, lens).to(torch.int32)   # some end
        pool.trim(lens)
        lists.plan(lens.tolist(), [0] * B)
        assert pool.held.tolist() == [len(x) for x in lists.tables]
    assert pool.status() == [] and cache.status() == []


def make(device_pages, batch=3, n_pages=18):
    w = workload("tiny").with_(batch=batch, prompt_len=(9, 40))
    W = make_weights(w)
    dec = PagedDecoder(w.shape, DeviceWeights.from_host(W, "f32"), split_k=w.split_k, k_spec=w.k_spec, max_seqs=batch,
                       n_pages=n_pages, max_seq_len=96, lora_gamma=w.lora_gamma, page_tokens=16, device_pages=device_pages)
    return w, W, dec


def sampling(seed, **kw):
    return Sampling(generator=torch.Generator(device="cuda").manual_seed(seed), **kw)


@pytest.mark.parametrize("speculative", [True, False])
def test_greedy_settings_give_the_greedy_tokens(speculative):
    """Temperature 0 and top_k 1 sample the greedy token, whatever hands out the pages."""
    w, _, dec = make(False)
    prompts = make_prompts(w)
    want = dec.generate(prompts, 20, speculative)
    for device_pages in (False, True):
        for kw in (dict(temperature=0.0), dict(top_k=1)):
            _, _, d = make(device_pages)
            assert d.generate(prompts, 20, speculative, sampling(3, **kw)) == want
    _, _, d = make(True)
    assert d.generate(prompts, 20, speculative) == want


@pytest.mark.parametrize("speculative", [True, False])
def test_sampled_tokens_are_among_the_likeliest(speculative):
    """Every token drawn with top_k 3 has one of the three largest logits of the 64-bit oracle, or is within the slack
    that int8 keys and values give the greedy tests; the same seed draws the same tokens, another one others."""
    w, W, dec = make(True)
    prompts = make_prompts(w)
    tokens, mat = dec.generate(prompts, 24, speculative, sampling(1, temperature=1.5, top_k=3))
    assert all(c.status() == [] for c in dec.caches) and dec.pool.status() == []
    model = OracleModel(W, w.shape, w.lora_gamma)
    for p, out in zip(prompts, tokens):
        z = teacher_forced_logits(model, np.concatenate([p, out[:-1]]))[len(p) - 1:]
        gap = np.sort(z, -1)[:, -3] - z[np.arange(len(out)), out]
        assert (gap <= 0.15 * z.std(-1)).all(), (gap / z.std(-1)).max()
    if speculative:
        assert 0 <= mat <= w.k_spec
    again = [make(True)[2].generate(prompts, 24, speculative, sampling(s, temperature=1.5, top_k=3))[0] for s in (1, 2)]
    assert again[0] == tokens and again[1] != tokens


def test_a_drafter_that_is_the_model_is_accepted():
    """All layers draft and the drafter's head is the model's: p = q but for rounding, so a draft is rejected only for
    u past 1 - 1e-4."""
    w = workload("tiny").with_(batch=2, prompt_len=(9, 20))
    W = make_weights(w)
    weights = DeviceWeights.from_host(W, "f32")
    weights.lora_a.zero_()
    dec = PagedDecoder(w.shape, weights, split_k=w.shape.n_layers, k_spec=4, max_seqs=2, n_pages=20, max_seq_len=96,
                       lora_gamma=w.lora_gamma, device_pages=True)
    _, mat = dec.generate(make_prompts(w), 24, True, sampling(5, temperature=1.0, top_p=0.9))
    assert mat > 3.8


def test_pages_of_the_pool_come_and_go():
    w, _, dec = make(True)
    prompts = make_prompts(w)
    first, _ = dec.generate(prompts, 12)
    assert dec.pages_in_use() == 18 - dec.pool.n_free.item() > 0
    for b in range(3):
        dec.release(b)
    assert dec.pages_in_use() == 0 and dec.lens.tolist() == [0, 0, 0] and bool((dec.table == -1).all())
    assert sorted(dec.pool.stack.tolist()) == list(range(18))
    again, _ = dec.generate(prompts, 12)
    assert again == first
    with pytest.raises(RuntimeError, match="max_seq_len"):
        dec.generate(prompts, 90)
    _, _, small = make(True, n_pages=2)
    with pytest.raises(RuntimeError, match="out of pages"):
        small.prefill(prompts)
    assert small.pages_in_use() == 0


def test_command(monkeypatch, capsys):
    monkeypatch.setattr("sys.argv", ["paged_decode", "--workload", "tiny", "--tokens", "8", "--batch", "2", "--temperature",
                                     "0.8", "--top-p", "0.9", "--top-k", "50", "--device-pages"])
    main()
    assert '"device_flags": []' in capsys.readouterr().out


def test_logits_that_are_no_numbers():
    """A step whose target gives no token says so (its sequence would never end)."""
    w, _, dec = make(True)
    tok = dec.prefill(make_prompts(w))
    lens = dec.lens.tolist()
    good = dec.verifier_logits
    dec.verifier_logits = lambda h: torch.where(torch.arange(len(good(h)), device="cuda")[:, None] < w.k_spec, torch.nan, good(h))
    with pytest.raises(RuntimeError, match="no token"):
        dec.step(tok, sampling=sampling(1))
    assert dec.lens.tolist() == lens


@pytest.mark.parametrize("at", [0, 2])
def test_generated_tokens_that_are_none(at):
    """Without drafts too: the prompt's next token, or a later one, that no probability gives is an error, not a token."""
    w, _, dec = make(True)
    good, calls = dec.verifier_logits, []

    def logits(h):
        calls.append(len(h))
        z = good(h)
        return torch.where(torch.arange(len(z), device="cuda")[:, None] < 1, torch.nan, z) if len(calls) == at + 1 else z

    dec.verifier_logits = logits
    with pytest.raises(RuntimeError, match="no token"):
        dec.generate(make_prompts(w), 12, False, sampling(1))
    assert len(calls) == at + 1
