"""Self-speculative decoding over the 8-bit paged KV cache: the draft, verify
and commit step of Sec. 3.3 for a batch of sequences of any lengths, with
pages taken as sequences grow and given back by release().

    python -m paper_2510_05421_gb300.paged_decode --workload tiny --fmt int8
    python -m paper_2510_05421_gb300.paged_decode --temperature 0.8 --top-p 0.9 --device-pages

One PagedCache per layer, one page table and one `lens` for all of them: every
pass appends its rows behind lens and attends from there, so a rejected draft
costs nothing but lens staying where it is.  With `sampling`, drafts are drawn
from the drafter's probabilities (token_probs) and verified so that what is
committed is distributed as the model's own tokens (verify_drafts); with
`device_pages` a PagePool hands out the pages on the GPU.  Projections run
through linear_noalloc and attention through PagedCache; the glue between them
(norms, SwiGLU, argmax) is plain torch, so this shows how the calls go
together, not how fast a decoder on them can be.  The contiguous-cache
engine (DVIEngine) is the fast path of a fixed batch.
"""
from __future__ import annotations

import argparse
import json
from dataclasses import dataclass
from typing import List, Optional, Sequence

import numpy as np
import torch

from .dvi import DEV_BITS, DeviceWeights, linear_noalloc
from .paged import PagedCache, rotary_table
from .pages import PagePool
from .sampling import token_probs, verify_drafts

_ROWS = 256     # rows of one linear_noalloc call


def _linear(w: torch.Tensor, x: torch.Tensor) -> torch.Tensor:
    """x W^T, f32 rows in and out."""
    y = torch.empty(x.shape[0], w.shape[0], device=x.device)
    for r in range(0, x.shape[0], _ROWS):
        rc = linear_noalloc(w, x[r:r + _ROWS].contiguous(), y[r:r + _ROWS])
        if rc != 0:
            raise RuntimeError(f"linear_noalloc: status {rc}")
    return y


@dataclass
class Sampling:
    """How tokens are drawn (as in token_probs), and from which numbers."""
    temperature: float = 1.0
    top_k: int = 0
    top_p: float = 1.0
    generator: Optional[torch.Generator] = None

    def uniform(self, n: int, device) -> torch.Tensor:
        return torch.rand(n, device=device, generator=self.generator)

    def probs(self, logits: torch.Tensor, status: Optional[torch.Tensor] = None) -> torch.Tensor:
        return token_probs(logits, self.temperature, self.top_k, self.top_p, status=status)

    def draw(self, probs: torch.Tensor, status: Optional[torch.Tensor] = None) -> torch.Tensor:
        """A token of each row (-1 of a row without probabilities)."""
        n = probs.shape[0]
        none = probs.new_empty(0)
        return verify_drafts(probs, none.to(torch.int32), none, self.uniform(n, probs.device), status=status)[0][:, 0]


class PagedDecoder:
    """A layer-split decoder whose sequences live in a pool of 8-bit pages."""

    pool: Optional[PagePool] = None
    status_word: Optional[torch.Tensor] = None      # of the sampling calls

    def __init__(self, shape, weights: DeviceWeights, *, split_k: int, k_spec: int, max_seqs: int, n_pages: int,
                 max_seq_len: int, lora_gamma: float = 1.0, page_tokens: int = 16, fmt: str = "int8",
                 device="cuda", device_pages: bool = False):
        self.s, self.w = shape, weights
        self.split, self.K, self.gamma, self.P = split_k, k_spec, lora_gamma, page_tokens
        self.device = torch.device(device)
        self.caches = [PagedCache.create(n_pages, shape.n_kv_heads, shape.head_dim, page_tokens, fmt, device)
                       for _ in range(shape.n_layers)]
        self.rotary = rotary_table(max_seq_len, shape.head_dim, shape.rope_theta, device)
        self.qkv = [torch.cat([l["wq"], l["wk"], l["wv"]]) for l in weights.layers]
        self.gate_up = [torch.cat([l["w_gate"], l["w_up"]]) for l in weights.layers]
        # queries, keys and values travel in the weights' type
        self.dtype = weights.embed.dtype
        self.free = list(range(n_pages))
        self.held: List[List[int]] = [[] for _ in range(max_seqs)]
        self.host_lens = [0] * max_seqs
        self.max_seq_len = max_seq_len
        self.reserved = [0] * max_seqs      # positions that reserve() has pages for (with device_pages)
        width = -(-max_seq_len // page_tokens)
        if device_pages:
            self.pool = PagePool.create(n_pages, max_seqs, width, page_tokens, device)
            self.table = self.pool.table
        else:
            self.table = torch.full((max_seqs, width), -1, dtype=torch.int32, device=device)
        self.lens = torch.zeros(max_seqs, dtype=torch.int32, device=device)
        self.status_word = torch.zeros(1, dtype=torch.int32, device=device)

    def status(self) -> list:
        """Names of the DVI_DEV_* flags that the caches, the pool and the sampling calls have set since the last look
        (waits for the device), then cleared."""
        names = {f for c in [*self.caches, *([self.pool] if self.pool else [])] for f in c.status()}
        word = int(self.status_word.item())
        self.status_word.bitwise_and_(~word)
        return sorted(names | {name for bit, name in DEV_BITS.items() if word & bit})

    # -- pages ------------------------------------------------------------
    def reserve(self, rows: Sequence[int]):
        """Pages for rows[b] more positions of each sequence.  They stay its own, whatever calls come before its rows do,
        until release(b)."""
        self._hold(rows)
        if self.pool is not None:
            self.reserved = [max(r, len_ + n) for r, len_, n in zip(self.reserved, self.host_lens, rows)]

    def _hold(self, rows: Sequence[int]):
        """The same for the pass that follows at once."""
        if self.pool is not None:
            self._plan(rows)
            return
        for b, n in enumerate(rows):
            if self.host_lens[b] + n > self.max_seq_len:
                raise RuntimeError("a sequence would outgrow max_seq_len")
            need = -(-(self.host_lens[b] + n) // self.P) - len(self.held[b])
            if need <= 0:
                continue
            if need > len(self.free):
                raise RuntimeError("out of pages")
            new = [self.free.pop() for _ in range(need)]
            at = len(self.held[b])
            self.table[b, at:at + need] = torch.tensor(new, dtype=torch.int32).to(self.device)
            self.held[b] += new

    def _plan(self, rows: Sequence[int]):
        """The same on the GPU: what the plan will find follows from the lengths, without a look at the device.  A plan
        brings every sequence to its rows, so those that are reserved are among them."""
        if max(len_ + n for len_, n in zip(self.host_lens, rows)) > self.max_seq_len:
            raise RuntimeError("a sequence would outgrow max_seq_len")
        after = [max(r, len_ + n) for r, len_, n in zip(self.reserved, self.host_lens, rows)]
        if sum(-(-n // self.P) for n in after) > self.pool.n_pages:
            raise RuntimeError("out of pages")
        more = [n - len_ for n, len_ in zip(after, self.host_lens)]
        self.pool.plan(self.lens, torch.tensor(more, dtype=torch.int32).to(self.device))

    def release(self, b: int):
        """Sequence b is over: its pages go back."""
        self.host_lens[b] = 0
        self.lens[b] = 0
        if self.pool is not None:
            self.reserved[b] = 0
            self._plan([0] * len(self.host_lens))
            return
        self.free += self.held[b]
        self.held[b] = []
        self.table[b].fill_(-1)

    def pages_in_use(self) -> int:
        return sum(len(h) for h in self.held) if self.pool is None else int(self.pool.held.sum())

    def advance(self, rows: Sequence[int]):
        """Keep rows[b] of the rows appended behind lens."""
        self.host_lens = [a + n for a, n in zip(self.host_lens, rows)]
        self.lens.add_(torch.tensor(list(rows), dtype=torch.int32).to(self.device))

    # -- the decoder ------------------------------------------------------
    def _norm(self, x, gain):
        return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + self.s.rms_eps) * gain

    def layers(self, lo: int, hi: int, x: torch.Tensor, lens: torch.Tensor, row_start=None, max_rows=None):
        """Layers lo .. hi - 1 on f32 rows x behind lens (their keys and values are appended)."""
        s = self.s
        n, nq, nkv = x.shape[0], s.n_heads, s.n_kv_heads
        for i in range(lo, hi):
            w, cache = self.w.layers[i], self.caches[i]
            qkv = _linear(self.qkv[i], self._norm(x, w["attn_norm"])).to(self.dtype).view(n, nq + 2 * nkv, s.head_dim)
            q, k, v = qkv[:, :nq], qkv[:, nq:nq + nkv], qkv[:, nq + nkv:]
            q = cache.append(self.table, lens, k, v, q=q, rotary=self.rotary, row_start=row_start, max_rows=max_rows)
            o = cache.attend(self.table, lens, q, row_start=row_start, max_rows=max_rows)
            x = x + _linear(w["wo"], o.float().view(n, nq * s.head_dim))
            g, u = _linear(self.gate_up[i], self._norm(x, w["ffn_norm"])).chunk(2, -1)
            x = x + _linear(w["w_down"], torch.nn.functional.silu(g) * u)
        return x

    def drafter_logits(self, h):
        u = self._norm(h, self.w.final_norm)
        z = _linear(self.w.draft_head, u)
        if self.w.lora_a.numel():
            z = z + self.gamma * (u @ self.w.lora_b.T) @ self.w.lora_a.T
        return z

    def verifier_logits(self, h):
        return _linear(self.w.lm_head, self._norm(h, self.w.final_norm))

    def embed(self, tokens: torch.Tensor):
        # (a draft that is none, -1, stands for token 0: it is rejected, and no row behind it counts)
        return self.w.embed[tokens.long().clamp_min(0)].float()

    # -- calls ------------------------------------------------------------
    def prefill(self, prompts: Sequence[np.ndarray], sampling: Optional[Sampling] = None) -> torch.Tensor:
        """The prompts, one for each slot, in one ragged pass behind what the sequences hold; the greedy (or sampled) token
        after each (pending, in no cache yet).  A slot whose prompt is empty takes no rows, and its token is -1, as is a
        sampled one where no token has a probability above 0 (logits that are no numbers)."""
        if len(prompts) != len(self.host_lens):
            raise ValueError(f"prefill: {len(prompts)} prompts for {len(self.host_lens)} slots")
        rows = [len(p) for p in prompts]
        if not any(rows):
            return torch.full((len(rows),), -1, dtype=torch.int32, device=self.device)
        self._hold(rows)
        start = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        row_start = torch.from_numpy(start).to(self.device)
        tokens = torch.from_numpy(np.concatenate(prompts).astype(np.int32)).to(self.device)
        h = self.layers(0, self.s.n_layers, self.embed(tokens), self.lens, row_start, max(rows))
        self.advance(rows)
        some = row_start.diff() > 0
        last = torch.where(some, row_start[1:] - 1, 0).long()
        return torch.where(some, self._choose(self.verifier_logits(h[last]), sampling), -1)

    def _choose(self, logits: torch.Tensor, sampling: Optional[Sampling]) -> torch.Tensor:
        """The greedy token of each row, or a sampled one."""
        if sampling is None:
            return logits.argmax(-1).to(torch.int32)
        return sampling.draw(sampling.probs(logits, self.status_word), self.status_word)

    @staticmethod
    def _some_token(what: str, got: Sequence[int]):
        """Refuses the -1 of a row that gave no token."""
        if min(got, default=0) < 0:
            raise RuntimeError(f"{what}: no token has a probability above 0 (logits that are no numbers)")

    @staticmethod
    def _has_token(what: str, pending: torch.Tensor):
        """Refuses a pending token of -1 (waits for the device)."""
        if bool((pending < 0).any()):
            raise ValueError(f"{what}: a sequence that takes part has no pending token")

    def _taking_part(self, live: Optional[Sequence[int]]):
        """The sequences of a pass (by default those that hold rows), where they lie in tensors of all sequences and
        the row starts of one row each; both None where every sequence takes part."""
        B = len(self.host_lens)
        live = [b for b in range(B) if self.host_lens[b]] if live is None else sorted(set(live))
        if len(live) == B:
            return live, None, None
        takes = [int(b in live) for b in range(B)]
        start = torch.tensor([0] + np.cumsum(takes).tolist(), dtype=torch.int32).to(self.device)
        return live, torch.tensor(live, dtype=torch.long).to(self.device), start

    def _spread(self, at, x: torch.Tensor, rest: Optional[torch.Tensor] = None):
        """x [sequences that took part, ...] among all of them; the others have rest, or 0."""
        if at is None:
            return x
        full = x.new_zeros((len(self.host_lens), *x.shape[1:])) if rest is None else rest.clone()
        return full.index_copy_(0, at, x)

    def step(self, pending: torch.Tensor, live: Optional[Sequence[int]] = None, sampling: Optional[Sampling] = None):
        """K greedy draft passes, one verify pass over the K rows, the longest agreeing prefix and the correction, of
        the sequences in `live` (by default those that hold rows: a released one takes none).  With `sampling` the drafts
        are drawn from the drafter's probabilities and verified against the model's.
        Returns (committed tokens [B, K], how many of them, how many drafts agreed, the new pending tokens); the
        sequences that took no part have 0 of them and their pending token as it was.  One that takes part without a
        pending token (-1) is a ValueError."""
        live, at, start = self._taking_part(live)
        n_live, K = len(live), self.K
        if n_live == 0:
            none = torch.zeros(len(self.host_lens), dtype=torch.long, device=self.device)
            return torch.zeros(len(none), K, dtype=torch.int32, device=self.device), none, none.clone(), pending
        tok = pending if at is None else pending[at]
        self._has_token("step", tok)
        self._hold([K if b in live else 0 for b in range(len(self.host_lens))])
        hs, drafts, drawn_from = [], [], []
        for j in range(K):
            h = self.layers(0, self.split, self.embed(tok), self.lens + j, start, 1)
            hs.append(h)
            z = self.drafter_logits(h)
            if sampling is None:
                tok = z.argmax(-1).to(torch.int32)
            else:
                drawn_from.append(sampling.probs(z, self.status_word))
                tok = sampling.draw(drawn_from[-1], self.status_word)
            drafts.append(tok)
        rows = torch.stack(hs, 1).reshape(n_live * K, -1)                # sequence after sequence
        h = self.layers(self.split, self.s.n_layers, rows, self.lens, None if start is None else start * K, K)
        t = torch.stack(drafts, 1)
        if sampling is None:
            y = self.verifier_logits(h).argmax(-1).to(torch.int32).view(n_live, K)
            m = (t == y).int().cumprod(1).sum(1)
            n = (m + 1).clamp_max(K)
            out = torch.where(torch.arange(K, device=self.device) < m[:, None], t, y)
        else:
            q = torch.stack(drawn_from, 1).view(n_live * K, -1)
            out, n, m = verify_drafts(sampling.probs(self.verifier_logits(h), self.status_word), t.view(-1),
                                      sampling.uniform(n_live * K, self.device), sampling.uniform(n_live, self.device),
                                      draft=q, max_drafts=K, bonus=False, status=self.status_word)
            n, m = n.long(), m.long()
        new_pending = out.gather(1, (n - 1).clamp_min(0).long()[:, None]).squeeze(1)
        n = self._spread(at, n)
        kept = n.tolist()
        self._some_token("step", [kept[b] - 1 for b in live])
        self.advance(kept)
        return self._spread(at, out), n, self._spread(at, m), self._spread(at, new_pending, pending)

    def ar_step(self, pending: torch.Tensor, live: Optional[Sequence[int]] = None,
                sampling: Optional[Sampling] = None) -> torch.Tensor:
        """One greedy (or sampled) token of the whole model for the sequences in `live` (by default those that hold rows);
        the others' pending tokens stay.  One that takes part without a pending token (-1) is a ValueError."""
        live, at, start = self._taking_part(live)
        if not live:
            return pending
        tok = pending if at is None else pending[at]
        self._has_token("ar_step", tok)
        takes = [int(b in live) for b in range(len(self.host_lens))]
        self._hold(takes)
        h = self.layers(0, self.s.n_layers, self.embed(tok), self.lens, start, 1)
        self.advance(takes)
        return self._spread(at, self._choose(self.verifier_logits(h), sampling), pending)

    def generate(self, prompts: Sequence[np.ndarray], n_gen: int, speculative: bool = True,
                 sampling: Optional[Sampling] = None):
        """n_gen tokens of each prompt, and the mean accepted length (None without speculation).  A sequence that has its
        tokens takes no more rows; its pages stay its own until release()."""
        if not all(len(p) for p in prompts):
            raise ValueError("generate: an empty prompt has no next token")
        tok = self.prefill(prompts, sampling)
        out = [[t] for t in tok.tolist()]
        self._some_token("generate", [t for t, in out])
        agreed = steps = 0
        while live := [b for b, o in enumerate(out) if len(o) < n_gen]:
            if speculative:
                ids, n, m, tok = self.step(tok, live, sampling)
                for o, row, c in zip(out, ids.tolist(), n.tolist()):
                    o.extend(row[:c])
                agreed += int(m.sum())
            else:
                tok = self.ar_step(tok, live, sampling)
                new = tok.tolist()
                self._some_token("generate", [new[b] for b in live])
                for b in live:
                    out[b].append(new[b])
            steps += len(live)
        return [o[:n_gen] for o in out], agreed / max(1, steps) if speculative else None


def run(workload_name: str, fmt: str, n_gen: int, page_tokens: int, batch: int, temperature: Optional[float] = None,
        top_k: int = 0, top_p: float = 1.0, seed: int = 0, device_pages: bool = False):
    from workloads import make_prompts, make_weights, workload

    w = workload(workload_name)
    if batch:
        w = w.with_(batch=batch, prompt_len=(max(1, w.prompt_len[0] // 2), w.prompt_len[1]))
    prompts = make_prompts(w)
    longest = max(len(p) for p in prompts) + n_gen + 2 * w.k_spec + 1
    dec = PagedDecoder(w.shape, DeviceWeights.from_host(make_weights(w), w.dtype), split_k=w.split_k, k_spec=w.k_spec,
                       max_seqs=w.batch, n_pages=w.batch * (-(-longest // page_tokens)), max_seq_len=longest,
                       lora_gamma=w.lora_gamma, page_tokens=page_tokens, fmt=fmt, device_pages=device_pages)
    sampling = None
    if temperature is not None:
        sampling = Sampling(temperature, top_k, top_p, torch.Generator(device="cuda").manual_seed(seed))
    tokens, mat = dec.generate(prompts, n_gen, sampling=sampling)
    return dict(workload=w.name, fmt=fmt, page_tokens=page_tokens, mean_accepted=mat, device_flags=dec.status(),
                pages_in_use=dec.pages_in_use(), tokens=[t[:8] for t in tokens])


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--workload", default="tiny")
    ap.add_argument("--fmt", default="int8", choices=("int8", "e4m3"))
    ap.add_argument("--tokens", type=int, default=32)
    ap.add_argument("--page-tokens", type=int, default=16)
    ap.add_argument("--batch", type=int, default=0, help="sequences of unequal prompts (0: the workload's batch)")
    ap.add_argument("--temperature", type=float, help="sample at this temperature (default: greedy)")
    ap.add_argument("--top-k", type=int, default=0)
    ap.add_argument("--top-p", type=float, default=1.0)
    ap.add_argument("--seed", type=int, default=0)
    ap.add_argument("--device-pages", action="store_true", help="plan the pages on the GPU")
    a = ap.parse_args()
    print(json.dumps(run(a.workload, a.fmt, a.tokens, a.page_tokens, a.batch, a.temperature, a.top_k, a.top_p, a.seed,
                         a.device_pages)))


if __name__ == "__main__":
    main()
