"""token_probs writes over a tensor of autograd's: a backward pass that has saved what it held fails, instead of going on
with probabilities in its place."""
import pytest
import torch

from paper_2510_05421_gb300 import sampling, token_probs


def saved(device):
    """Logits that a backward pass has saved, and what it leads to."""
    x = torch.linspace(-1, 1, 12, device=device).view(3, 4).requires_grad_()
    logits = x * 2
    return x, logits, logits.square().sum()


def check(device, call):
    x, logits, loss = saved(device)
    with pytest.raises(ValueError):
        call(logits, out=logits[:2])
    loss.backward()                             # (nothing was written)
    assert torch.equal(x.grad, 8 * x.detach())
    for detached in (False, True):
        x, logits, loss = saved(device)
        call(logits.detach(), out=logits.detach() if detached else logits)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
    x, logits, loss = saved(device)
    call(logits)                                # (its own output)
    loss.backward()
    with torch.inference_mode():
        out = torch.zeros(3, 4, device=device)
    call(logits.detach(), out=out)              # has no version: written, as ever
    assert torch.allclose(out.sum(1), torch.ones(3, device=device))


def test_the_version_goes_up(monkeypatch):
    """Around a stand-in for the module's call."""
    class Calls:
        @staticmethod
        def probs(logits, temperature, top_k, top_p, out, status, stream):
            if out is not None and out.shape != logits.shape:
                raise ValueError("out")
            p = logits.detach().softmax(-1)
            if out is None:
                return p
            out.detach().numpy()[:] = p.numpy()     # (unseen by autograd)
            return out
    monkeypatch.setattr(sampling, "_calls", Calls)
    monkeypatch.setattr(sampling, "_device_of", lambda what, t: 0)
    monkeypatch.setattr(sampling, "_current", lambda: 0)
    monkeypatch.setattr(sampling, "_raw_stream", lambda index: 0)
    check("cpu", sampling.token_probs)


@pytest.mark.gpu
@pytest.mark.parametrize("other_stream", [False, True])
def test_on_the_gpu(other_stream):
    stream = torch.cuda.Stream() if other_stream else None
    check("cuda", lambda logits, **kw: token_probs(logits, stream=stream, **kw))
    torch.cuda.synchronize()
