"""What reserve() promises, with pages from the host and from a pool: a sequence's pages stay its own until release,
whatever is called before its rows come."""
import numpy as np
import pytest
import torch

import sampling_ref as ref
from test_paged_decoder import P, V, Decoder, chain, prompts


class Pool:
    """PagePool's definition on lists."""

    def __init__(self, n_pages, slots, width):
        self.n_pages, self.lists = n_pages, ref.Pool(n_pages, slots, width, P)
        self.table = torch.full((slots, width), -1, dtype=torch.int32)

    def plan(self, lens, rows=0):
        rows = [rows] * len(lens) if isinstance(rows, int) else rows.tolist()
        assert not self.lists.plan(lens.tolist(), rows)[3]
        self.table.copy_(torch.from_numpy(self.lists.table()))

    def trim(self, lens):
        self.plan(lens)

    @property
    def held(self):
        return torch.tensor([len(t) for t in self.lists.tables])


def make(device_pages, slots=2, room=100, n_pages=14):
    dec = Decoder(slots, room, n_pages)
    if device_pages:
        dec.reserved = [0] * slots
        dec.pool = Pool(n_pages, slots, dec.table.shape[1])
        dec.table = dec.pool.table
    return dec


def rows(dec, counts):
    """A pass of counts[b] rows (Decoder.layers looks whether their pages are held)."""
    start = torch.tensor(np.concatenate([[0], np.cumsum(counts)]))
    dec.layers(0, 1, torch.zeros(sum(counts), V), dec.lens, start, max(counts))


@pytest.mark.parametrize("device_pages", [False, True])
class TestReserve:
    def test_one_after_the_other(self, device_pages):
        dec = make(device_pages)
        dec.reserve([40, 0])
        dec.reserve([0, 40])
        rows(dec, [40, 40])

    def test_a_release_between(self, device_pages):
        dec = make(device_pages)
        dec.prefill(prompts(2, 4))
        dec.reserve([40, 0])
        dec.release(1)
        rows(dec, [40, 0])
        assert dec.pages_in_use() == 3

    def test_steps_of_others_between(self, device_pages):
        dec = make(device_pages, n_pages=12)
        tok = dec.prefill(prompts(2, 4))
        dec.reserve([50, 0])
        for _ in range(5):
            tok = dec.step(tok, [1])[3]
            tok = dec.ar_step(tok, [1])
        rows(dec, [50, 0])

    def test_some_of_the_rows_first(self, device_pages):
        dec = make(device_pages)
        dec.reserve([40, 0])
        rows(dec, [20, 0])
        dec.advance([20, 0])
        dec.reserve([0, 4])
        rows(dec, [20, 4])

    def test_fewer_later(self, device_pages):
        dec = make(device_pages)
        dec.reserve([40, 4])
        dec.reserve([4, 0])
        rows(dec, [40, 4])
        dec.release(0)
        dec.release(1)
        assert dec.pages_in_use() == 0

    def test_too_many(self, device_pages):
        dec = make(device_pages, n_pages=4)
        dec.reserve([40, 0])
        with pytest.raises(RuntimeError, match="out of pages"):
            dec.reserve([0, 40])
        with pytest.raises(RuntimeError, match="max_seq_len"):
            dec.reserve([101, 0])
        rows(dec, [40, 0])
        dec.release(0)
        dec.reserve([0, 40])
        rows(dec, [0, 40])


def test_pages_of_rejected_rows_go_round():
    """Pages from the pool that a pass took and its rejected rows did not keep are there for other sequences."""
    dec = make(True, n_pages=3)
    tok = dec.prefill(prompts(3, 5))
    dec.advance([14 - n for n in dec.host_lens])
    for live in ([0], [1]):                     # each takes a second page and keeps one row, in the first
        tok = dec.step(tok, live)[3]
        assert dec.pages_in_use() == 3
    assert dec.host_lens == [15, 15] and tok.tolist() == [chain(3, 2)[1], chain(5, 2)[1]]
