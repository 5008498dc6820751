"""PagedDecoder's bookkeeping without a GPU, over a stand-in for the layers: which sequences a pass takes, what they may
need of pages and positions, and what they commit.  In the stand-in's language an even token t is followed by t + 2, and
the drafter says so; an odd one by t + 4, where the drafter says t + 2 and is always rejected."""
import numpy as np
import pytest
import torch

from paper_2510_05421_gb300.paged_decode import PagedDecoder

V, P, K, SPLIT, LAYERS = 400, 16, 4, 1, 2


class Shape:
    n_layers = LAYERS


class Decoder(PagedDecoder):
    """The layers see nothing and pass on which token each row had; what a pass takes is noted."""

    def __init__(self, slots, max_seq_len, n_pages):
        self.s, self.split, self.K, self.P = Shape, SPLIT, K, P
        self.device = torch.device("cpu")
        self.caches = []
        self.free = list(range(n_pages))
        self.held = [[] for _ in range(slots)]
        self.host_lens = [0] * slots
        self.max_seq_len = max_seq_len
        self.table = torch.full((slots, -(-max_seq_len // P)), -1, dtype=torch.int32)
        self.lens = torch.zeros(slots, dtype=torch.int32)
        self.rows = []

    def embed(self, tokens):
        return torch.nn.functional.one_hot(tokens.long(), V).float()

    def layers(self, lo, hi, x, lens, row_start=None, max_rows=None):
        B = len(self.host_lens)
        counts = [x.shape[0] // B] * B if row_start is None else row_start.diff().tolist()
        assert sum(counts) == x.shape[0] and (max_rows is None or max(counts) <= max_rows)
        for b, n in enumerate(counts):
            # every row has a position, and its page is held
            assert int(lens[b]) + n <= self.max_seq_len
            for p in range(int(lens[b]), int(lens[b]) + n):
                assert int(self.table[b, p // P]) >= 0
        self.rows.append(counts)
        return x

    def drafter_logits(self, h):
        return torch.roll(h, 2, -1)

    def verifier_logits(self, h):
        odd = h.argmax(-1) % 2 == 1
        return torch.where(odd[:, None], torch.roll(h, 4, -1), torch.roll(h, 2, -1))


def prompts(*last):
    return [np.array([9, 9, t], np.int32)[-(1 + t % 3):] for t in last]


def chain(t, n):
    step = 4 if t % 2 else 2
    return [t + step * (i + 1) for i in range(n)]


@pytest.mark.parametrize("first", [(2, 3), (3, 2), (2, 3, 4, 5)])
@pytest.mark.parametrize("speculative", [True, False])
def test_sequences_of_unequal_acceptance(first, speculative):
    """A sequence that has its tokens takes no more rows, while one whose drafts all fail goes on: what both need is
    bounded by their own lengths."""
    n_gen, p = 40, prompts(*first)
    room = max(len(x) for x in p) + n_gen + 2 * K + 1
    dec = Decoder(len(first), room, len(first) * -(-room // P))
    tokens, mean = dec.generate(p, n_gen, speculative)
    assert tokens == [chain(t, n_gen) for t in first]
    for x, n in zip(p, dec.host_lens):
        assert len(x) + n_gen - 1 <= n < len(x) + n_gen - 1 + K
    if speculative:
        fast = -(-(n_gen - 1) // K)
        assert sum(c[first.index(2)] > 0 for c in dec.rows[1:]) == fast * (K + 1)
        # per step of a sequence: all K drafts agree, or none
        evens = sum(t % 2 == 0 for t in first)
        assert mean == pytest.approx(evens * fast * K / (evens * fast + (len(first) - evens) * (n_gen - 1)))


def test_released_sequences_take_no_rows():
    p = prompts(2, 3, 4)
    dec = Decoder(3, 64, 12)
    tok = dec.prefill(p)
    assert tok.tolist() == [4, 7, 6]
    dec.release(1)
    free = len(dec.free)
    for _ in range(3):
        out, n, m, new = dec.step(tok)
        assert n.tolist() == [K, 0, K] and m.tolist() == [K, 0, K] and new[1] == tok[1]
        assert out[0].tolist() == chain(int(tok[0]), K) and out[2].tolist() == chain(int(tok[2]), K)
        tok = new
    tok = dec.ar_step(tok)
    assert tok[0] == 4 + 2 * 3 * K + 2 and tok[1] == 7
    assert dec.held[1] == [] and dec.host_lens[1] == 0 and dec.lens.tolist()[1] == 0
    assert len(dec.free) <= free and all(c[1] == 0 for c in dec.rows[1:])
    for b in (0, 2):
        dec.release(b)
    assert sorted(dec.free) == list(range(12))
    out, n, m, new = dec.step(tok)
    assert n.tolist() == [0, 0, 0] and torch.equal(new, tok) and torch.equal(dec.ar_step(tok), tok)


def test_prompts_that_do_not_fit_the_slots_are_refused():
    """Before any page is taken."""
    dec = Decoder(2, 64, 8)
    one = np.array([2], np.int32)
    for bad in ([one], [one] * 3, []):
        with pytest.raises(ValueError):
            dec.prefill(bad)
        with pytest.raises(ValueError):
            dec.generate(bad, 4)
    assert len(dec.free) == 8 and dec.host_lens == [0, 0] and dec.rows == []


def test_empty_prompts():
    """A slot without a prompt gets no rows and no token; the others' tokens are theirs, and a slot filled later joins."""
    empty = np.zeros(0, np.int32)
    dec = Decoder(3, 64, 12)
    assert dec.prefill([empty, np.array([5, 8], np.int32), empty]).tolist() == [-1, 10, -1]
    assert dec.lens.tolist() == [0, 2, 0] and dec.held[0] == [] and dec.held[2] == []
    first = dec.prefill([np.array([3], np.int32), empty, empty])
    assert first.tolist() == [7, -1, -1] and dec.lens.tolist() == [1, 2, 0]
    assert dec.prefill([empty] * 3).tolist() == [-1, -1, -1]
    out, n, _, _ = dec.step(torch.tensor([7, 10, -1], dtype=torch.int32))
    assert n.tolist() == [1, K, 0] and out[0, 0] == 11 and out[1].tolist() == chain(10, K)
    with pytest.raises(ValueError):
        dec.generate([empty, np.array([3], np.int32), empty], 4)
    assert dec.host_lens == [2, 6, 0]
