"""PagedDecoder says what its sampling calls have flagged."""
import pytest
import torch

from paper_2510_05421_gb300 import DeviceWeights
from paper_2510_05421_gb300.paged_decode import PagedDecoder, Sampling, run
from workloads import make_prompts, make_weights, workload

pytestmark = pytest.mark.gpu


def make(**kw):
    w = workload("tiny").with_(batch=2, prompt_len=(9, 20))
    dec = PagedDecoder(w.shape, DeviceWeights.from_host(make_weights(w), "f32"), split_k=w.split_k, k_spec=w.k_spec,
                       max_seqs=2, n_pages=20, max_seq_len=96, lora_gamma=w.lora_gamma, **kw)
    return dec, make_prompts(w), Sampling(generator=torch.Generator(device="cuda").manual_seed(1))


def odd(logits, what):
    """The same logits with some of a row's that are no numbers; numbers are left."""
    def f(h):
        z = logits(h).clone()
        z[0, 1::7] = what
        return z
    return f


@pytest.mark.parametrize("where", ["prefill", "drafter", "verifier", "ar_step"])
@pytest.mark.parametrize("device_pages", [False, True])
def test_logits_that_are_partly_no_numbers(where, device_pages):
    dec, prompts, sampling = make(device_pages=device_pages)
    verifier = dec.verifier_logits
    if where == "prefill":
        dec.verifier_logits = odd(verifier, torch.nan)
    tok = dec.prefill(prompts, sampling)
    assert dec.status() == (["NONFINITE"] if where == "prefill" else [])
    dec.verifier_logits = verifier
    if where == "drafter":
        dec.drafter_logits = odd(dec.drafter_logits, torch.inf)
    elif where != "prefill":
        dec.verifier_logits = odd(verifier, torch.nan)
    if where == "ar_step":
        dec.ar_step(tok, sampling=sampling)
    else:
        dec.step(tok, sampling=sampling)
    assert dec.status() == ([] if where == "prefill" else ["NONFINITE"])
    assert dec.status() == []


def test_a_drafter_without_tokens():
    """Rows of the drafter that give no token: what it drafts is none (flagged, rejected), the model's token comes."""
    dec, prompts, sampling = make()
    tok = dec.prefill(prompts, sampling)
    dec.drafter_logits = lambda h: torch.full((len(h), dec.s.vocab), torch.nan, device="cuda")
    _, n, m, _ = dec.step(tok, sampling=sampling)
    assert n.tolist() == [1, 1] and m.tolist() == [0, 0]
    assert dec.status() == ["BAD_TOKEN", "NONFINITE"]


def test_command(monkeypatch):
    assert run("tiny", "int8", 8, 16, 2, temperature=0.8)["device_flags"] == []
    good = PagedDecoder.verifier_logits
    monkeypatch.setattr(PagedDecoder, "verifier_logits", lambda self, h: odd(lambda h: good(self, h), torch.nan)(h))
    assert run("tiny", "int8", 8, 16, 2, temperature=0.8)["device_flags"] == ["NONFINITE"]
