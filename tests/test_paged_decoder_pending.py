"""PagedDecoder's calls on sequences without a pending token, over the stand-in for the layers of test_paged_decoder."""
import pytest
import torch

from test_paged_decoder import Decoder, prompts


@pytest.mark.parametrize("call", ["step", "ar_step"])
@pytest.mark.parametrize("live", [None, [1], [0, 1]])
def test_a_sequence_without_a_pending_token(call, live):
    """What prefill (an empty prompt) or a sampled call (no token has a probability) leaves as -1 is no token to go on
    from: refused before anything changes.  Of a sequence that takes no part it may stand there."""
    dec = Decoder(2, 64, 8)
    tok = dec.prefill(prompts(2, 4))
    lens, table, passes = dec.lens.tolist(), dec.table.clone(), len(dec.rows)
    with pytest.raises(ValueError, match="no pending token"):
        getattr(dec, call)(torch.where(torch.arange(2) == 1, -1, tok), live)
    assert dec.lens.tolist() == dec.host_lens == lens and torch.equal(dec.table, table) and len(dec.rows) == passes
    getattr(dec, call)(torch.where(torch.arange(2) == 1, -1, tok), [0])
    getattr(dec, call)(tok, live)


def test_an_empty_slot_is_taken_along():
    dec = Decoder(2, 64, 8)
    tok = dec.prefill([prompts(2)[0], prompts(2)[0][:0]])
    assert tok.tolist() == [4, -1]
    for call in (dec.step, dec.ar_step):
        with pytest.raises(ValueError, match="no pending token"):
            call(tok, [0, 1])
        call(tok)
