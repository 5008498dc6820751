"""Binding of sampled speculative decoding (include/dvi.h): the probabilities
of logits and the verification of drafted tokens against them.  Argument
checks and marshalling only (csrc/sampling_py.c); the tensors are the
caller's, the random numbers inputs, and every call enqueues on the caller's
current stream (or the one it names)."""
from __future__ import annotations

import ctypes
from typing import Optional, Tuple, Union

import torch

from .dvi import DVIError, lib
from .paged import _empty_strided, _raw_stream, elsewhere

_calls = None
# (the call behind torch.cuda.current_device, without a look at whether CUDA is there)
_current = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _empty(size, stride, dtype):
    """A tensor on the current device, where torch has no shorter way."""
    return torch.empty_strided(size, stride, dtype=dtype, device="cuda")


def _module():
    """The CPython module with the library's entry points; raises if it was not built (there is no fallback)."""
    global _calls
    if _calls is None:
        L = lib()
        try:
            from . import _sampling
        except ImportError as e:
            raise RuntimeError("_sampling.so is missing: build it with `python -m paper_2510_05421_gb300.build`") from e
        at = (ctypes.cast(f, ctypes.c_void_p).value for f in (L.dvi_token_probs, L.dvi_verify_drafts, L.dvi_paged_plan))
        _sampling.init(*at, torch.int32, torch.int64, torch.float32, torch.bfloat16, _empty_strided or _empty, DVIError)
        _calls = _sampling
    return _calls


def _device_of(what: str, t: torch.Tensor) -> int:
    index = t.get_device() if isinstance(t, torch.Tensor) else -1
    if index < 0:
        raise ValueError(f"{what}: not a tensor on a CUDA device")
    return index


def token_probs(logits: torch.Tensor, temperature: Union[float, torch.Tensor] = 1.0,
                top_k: Union[int, torch.Tensor] = 0, top_p: Union[float, torch.Tensor] = 1.0,
                out: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Probabilities f32 [n, vocab] of logits [n, vocab] (f32 or bf16; rows may lie apart): softmax(logits /
    temperature) over the top_k largest logits (0: all) and of those the fewest whose probabilities sum to top_p
    (at least one), 0 elsewhere; equal logits count in order of their index.  Temperature 0: 1 at the first of the
    largest.  A row of -inf alone gets zeros.

    Settings are numbers or tensors with one for each row (f32, int32, f32 [n]).  NaN logits count as -inf, +inf as
    the largest number; status (int32 [1], or None) gets DVI_DEV_NONFINITE then, and DVI_DEV_TIMEOUT where a bounded wait
    of the device ran out, whose row gets zeros.  `out` may be the logits (f32); one that
    overlaps them in another way is refused.  No gradient passes through; that `out` was written in place is known to
    autograd, which refuses a backward pass that has saved what it held."""
    index = _device_of("token_probs: logits", logits)
    if stream is not None or _current() != index:
        return elsewhere(index, stream, (), token_probs, (logits, temperature, top_k, top_p, out, status),
                         "the logits' device")
    got = (_calls or _module()).probs(logits, temperature, top_k, top_p, out, status, _raw_stream(index))
    if out is not None and not out.is_inference():
        torch.autograd.graph.increment_version(out)
    return got


def verify_drafts(target: torch.Tensor, draft_ids: torch.Tensor, u_accept: torch.Tensor, u_token: torch.Tensor,
                  draft: Optional[torch.Tensor] = None, draft_start: Optional[torch.Tensor] = None,
                  max_drafts: Optional[int] = None, bonus: bool = True, status: Optional[torch.Tensor] = None,
                  stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Verify the drafted tokens of n_seqs sequences so that what is committed is distributed as the target's own
    tokens: draft x_j is accepted while u_accept q_j(x_j) < p_j(x_j); behind the m accepted ones comes a token of
    max(p - q, 0) of the first rejected place, or (all accepted, bonus) of the bonus row, chosen by u_token.

    target: f32 [n_drafts + n_seqs * bonus, vocab], the rows p_j of a sequence's drafts and then its bonus row,
    sequence after sequence.  draft: f32 [n_drafts, vocab], the rows q_j the drafts were drawn from, or None for greedy
    drafts.  draft_ids: int32 [n_drafts]; with draft_start None every sequence has the same number, else sequence b has
    drafts draft_start[b] .. draft_start[b + 1] - 1 (int32 [n_seqs + 1]) and max_drafts bounds the most.  u_accept f32
    [n_drafts] and u_token f32 [n_seqs]: uniform in [0, 1).  With no drafts and a bonus row it samples a token a row.

    Returns (ids int32 [n_seqs, max_drafts + bonus], how many of them are committed, how many drafts were accepted);
    entries behind the committed ones are -1.  status (int32 [1], or None): DVI_DEV_BAD_TOKEN for a drafted id outside
    the vocabulary (rejected) and for starts that fall or lie outside the drafts (cut to them), DVI_DEV_NONFINITE for probabilities that are not finite (taken as 0) and rows that are
    zero everywhere (no token)."""
    index = _device_of("verify_drafts: target", target)
    if stream is not None or _current() != index:
        return elsewhere(index, stream, (), verify_drafts, (target, draft_ids, u_accept, u_token, draft, draft_start,
                                                            max_drafts, bonus, status), "the target's device")
    return (_calls or _module()).verify(target, draft_ids, u_accept, u_token, draft, draft_start, max_drafts, bonus,
                                        status, _raw_stream(index))
