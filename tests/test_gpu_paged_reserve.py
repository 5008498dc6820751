"""Pages reserved for several sequences one after the other, on the GPU as from the host: all rows of the pass that
follows are kept."""
import pytest
import torch

from paper_2510_05421_gb300 import DeviceWeights
from paper_2510_05421_gb300.paged_decode import PagedDecoder
from workloads import make_prompts, make_weights, workload

pytestmark = pytest.mark.gpu


def outputs(device_pages):
    w = workload("tiny").with_(batch=3, prompt_len=(9, 20))
    dec = PagedDecoder(w.shape, DeviceWeights.from_host(make_weights(w), "f32"), split_k=w.split_k, k_spec=w.k_spec,
                       max_seqs=3, n_pages=12, max_seq_len=64, lora_gamma=w.lora_gamma, device_pages=device_pages)
    dec.prefill(make_prompts(w))
    dec.reserve([20, 0, 0])
    dec.reserve([0, 20, 0])
    dec.release(2)
    tokens = torch.arange(40, device="cuda") * 7
    start = torch.tensor([0, 20, 40, 40], dtype=torch.int32, device="cuda")
    h = dec.layers(0, w.shape.n_layers, dec.embed(tokens), dec.lens, start, 20)
    assert dec.status() == []
    assert dec.pages_in_use() == sum(-(-(n + 20) // 16) for n in dec.host_lens[:2])
    return h


def test_reserved_rows_are_kept():
    want = outputs(False)
    assert bool(want.isfinite().all()) and torch.equal(outputs(True), want)
