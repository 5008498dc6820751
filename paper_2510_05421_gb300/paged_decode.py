"""Self-speculative decoding over the 8-bit paged KV cache: the draft, verify
and commit step of Sec. 3.3 for a batch of sequences of any lengths, with
pages taken as sequences grow and given back by release().

    python -m paper_2510_05421_gb300.paged_decode --workload tiny --fmt int8

One PagedCache per layer, one page table and one `lens` for all of them: every
pass appends its rows behind lens and attends from there, so a rejected draft
costs nothing but lens staying where it is.  Projections run through
linear_noalloc and attention through PagedCache; the glue between them
(norms, SwiGLU, argmax) is plain torch, so this shows how the calls go
together, not how fast a decoder on them can be.  The contiguous-cache
engine (DVIEngine) is the fast path of a fixed batch.
"""
from __future__ import annotations

import argparse
import json
from typing import List, Optional, Sequence

import numpy as np
import torch

from .dvi import DeviceWeights, linear_noalloc
from .paged import PagedCache, rotary_table

_ROWS = 256     # rows of one linear_noalloc call


def _linear(w: torch.Tensor, x: torch.Tensor) -> torch.Tensor:
    """x W^T, f32 rows in and out."""
    y = torch.empty(x.shape[0], w.shape[0], device=x.device)
    for r in range(0, x.shape[0], _ROWS):
        rc = linear_noalloc(w, x[r:r + _ROWS].contiguous(), y[r:r + _ROWS])
        if rc != 0:
            raise RuntimeError(f"linear_noalloc: status {rc}")
    return y


class PagedDecoder:
    """A layer-split decoder whose sequences live in a pool of 8-bit pages."""

    def __init__(self, shape, weights: DeviceWeights, *, split_k: int, k_spec: int, max_seqs: int, n_pages: int,
                 max_seq_len: int, lora_gamma: float = 1.0, page_tokens: int = 16, fmt: str = "int8",
                 device="cuda"):
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
        self.table = torch.full((max_seqs, -(-max_seq_len // page_tokens)), -1, dtype=torch.int32, device=device)
        self.lens = torch.zeros(max_seqs, dtype=torch.int32, device=device)

    # -- pages ------------------------------------------------------------
    def reserve(self, rows: Sequence[int]):
        """Pages for rows[b] more positions of each sequence."""
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

    def release(self, b: int):
        """Sequence b is over: its pages go back."""
        self.free += self.held[b]
        self.held[b] = []
        self.host_lens[b] = 0
        self.table[b].fill_(-1)
        self.lens[b] = 0

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
        return self.w.embed[tokens.long()].float()

    # -- calls ------------------------------------------------------------
    def prefill(self, prompts: Sequence[np.ndarray]) -> torch.Tensor:
        """The prompts, one for each slot, in one ragged pass behind what the sequences hold; the greedy token after each
        (pending, in no cache yet).  A slot whose prompt is empty takes no rows, and its token is -1."""
        if len(prompts) != len(self.host_lens):
            raise ValueError(f"prefill: {len(prompts)} prompts for {len(self.host_lens)} slots")
        rows = [len(p) for p in prompts]
        if not any(rows):
            return torch.full((len(rows),), -1, dtype=torch.int32, device=self.device)
        self.reserve(rows)
        start = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        row_start = torch.from_numpy(start).to(self.device)
        tokens = torch.from_numpy(np.concatenate(prompts).astype(np.int32)).to(self.device)
        h = self.layers(0, self.s.n_layers, self.embed(tokens), self.lens, row_start, max(rows))
        self.advance(rows)
        some = row_start.diff() > 0
        last = torch.where(some, row_start[1:] - 1, 0).long()
        return torch.where(some, self.verifier_logits(h[last]).argmax(-1).to(torch.int32), -1)

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

    def step(self, pending: torch.Tensor, live: Optional[Sequence[int]] = None):
        """K greedy draft passes, one verify pass over the K rows, the longest agreeing prefix and the correction, of
        the sequences in `live` (by default those that hold rows: a released one takes none).
        Returns (committed tokens [B, K], how many of them, how many drafts agreed, the new pending tokens); the
        sequences that took no part have 0 of them and their pending token as it was."""
        live, at, start = self._taking_part(live)
        n_live, K = len(live), self.K
        if n_live == 0:
            none = torch.zeros(len(self.host_lens), dtype=torch.long, device=self.device)
            return torch.zeros(len(none), K, dtype=torch.int32, device=self.device), none, none.clone(), pending
        self.reserve([K if b in live else 0 for b in range(len(self.host_lens))])
        hs, drafts = [], []
        tok = pending if at is None else pending[at]
        for j in range(K):
            h = self.layers(0, self.split, self.embed(tok), self.lens + j, start, 1)
            hs.append(h)
            tok = self.drafter_logits(h).argmax(-1).to(torch.int32)
            drafts.append(tok)
        rows = torch.stack(hs, 1).reshape(n_live * K, -1)                # sequence after sequence
        h = self.layers(self.split, self.s.n_layers, rows, self.lens, None if start is None else start * K, K)
        y = self.verifier_logits(h).argmax(-1).to(torch.int32).view(n_live, K)
        t = torch.stack(drafts, 1)
        m = (t == y).int().cumprod(1).sum(1)
        n = (m + 1).clamp_max(K)
        out = torch.where(torch.arange(K, device=self.device) < m[:, None], t, y)
        new_pending = out.gather(1, (n - 1).long()[:, None]).squeeze(1)
        n = self._spread(at, n)
        self.advance(n.tolist())
        return self._spread(at, out), n, self._spread(at, m), self._spread(at, new_pending, pending)

    def ar_step(self, pending: torch.Tensor, live: Optional[Sequence[int]] = None) -> torch.Tensor:
        """One greedy token of the whole model for the sequences in `live` (by default those that hold rows); the
        others' pending tokens stay."""
        live, at, start = self._taking_part(live)
        if not live:
            return pending
        takes = [int(b in live) for b in range(len(self.host_lens))]
        self.reserve(takes)
        tok = pending if at is None else pending[at]
        h = self.layers(0, self.s.n_layers, self.embed(tok), self.lens, start, 1)
        self.advance(takes)
        return self._spread(at, self.verifier_logits(h).argmax(-1).to(torch.int32), pending)

    def generate(self, prompts: Sequence[np.ndarray], n_gen: int, speculative: bool = True):
        """n_gen tokens of each prompt, and the mean accepted length (None without speculation).  A sequence that has its
        tokens takes no more rows; its pages stay its own until release()."""
        if not all(len(p) for p in prompts):
            raise ValueError("generate: an empty prompt has no next token")
        tok = self.prefill(prompts)
        out = [[int(t)] for t in tok]
        agreed = steps = 0
        while live := [b for b, o in enumerate(out) if len(o) < n_gen]:
            if speculative:
                ids, n, m, tok = self.step(tok, live)
                for o, row, c in zip(out, ids.tolist(), n.tolist()):
                    o.extend(row[:c])
                agreed += int(m.sum())
            else:
                tok = self.ar_step(tok, live)
                new = tok.tolist()
                for b in live:
                    out[b].append(new[b])
            steps += len(live)
        return [o[:n_gen] for o in out], agreed / max(1, steps) if speculative else None


def run(workload_name: str, fmt: str, n_gen: int, page_tokens: int, batch: int):
    from workloads import make_prompts, make_weights, workload

    w = workload(workload_name)
    if batch:
        w = w.with_(batch=batch, prompt_len=(max(1, w.prompt_len[0] // 2), w.prompt_len[1]))
    prompts = make_prompts(w)
    longest = max(len(p) for p in prompts) + n_gen + 2 * w.k_spec + 1
    dec = PagedDecoder(w.shape, DeviceWeights.from_host(make_weights(w), w.dtype), split_k=w.split_k, k_spec=w.k_spec,
                       max_seqs=w.batch, n_pages=w.batch * (-(-longest // page_tokens)), max_seq_len=longest,
                       lora_gamma=w.lora_gamma, page_tokens=page_tokens, fmt=fmt)
    tokens, mat = dec.generate(prompts, n_gen)
    flags = sorted({f for c in dec.caches for f in c.status()})
    return dict(workload=w.name, fmt=fmt, page_tokens=page_tokens, mean_accepted=mat, device_flags=flags,
                pages_in_use=sum(len(h) for h in dec.held), tokens=[t[:8] for t in tokens])


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--workload", default="tiny")
    ap.add_argument("--fmt", default="int8", choices=("int8", "e4m3"))
    ap.add_argument("--tokens", type=int, default=32)
    ap.add_argument("--page-tokens", type=int, default=16)
    ap.add_argument("--batch", type=int, default=0, help="sequences of unequal prompts (0: the workload's batch)")
    a = ap.parse_args()
    print(json.dumps(run(a.workload, a.fmt, a.tokens, a.page_tokens, a.batch)))


if __name__ == "__main__":
    main()
