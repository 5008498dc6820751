"""Sampled speculative decoding's operators as measurable cases: probabilities, verification, page plans.

A program that decodes with a temperature over the paged cache makes three
calls around each pass of the decoder.  Before it, the page plan: pages for
the rows that each sequence is about to append, taken from and given back to
a pool on the GPU, with row starts and slots (and behind it the plan again,
for the lengths that were kept).  After it, the probabilities of the logits
(temperature, top-k, top-p, one set for each row), and the verification of
the drafted tokens against them from given uniform numbers: accept length,
correction or bonus token.  The listed cases use the repository's decoders
(tiny: 1024 tokens in the vocabulary; 1B- and 7B-shaped: 32000) and a larger,
odd vocabulary; draw() spreads more over the same ranges.

Logits are normal with a few likely tokens in each row, drafts are drawn from
a drafter whose logits are the verifier's with noise on them.
"""
from __future__ import annotations

import math

import torch

own = False      # True: the library's operators; False: the same in elementary torch operations

DEV = "cuda"


def listed():
    return [
        # the next token's probabilities of the tiny f32 decoder, nothing cut off: the smallest, latency counts
        _probs("probs_tiny_token", 1, 1024, temperature=0.8),
        # the verify block (5 drafts and the bonus row) of one sequence on the 7B-shaped decoder, nucleus sampling
        _probs("probs_7b_block", 6, 32000, temperature=0.8, top_p=0.9),
        # the verify rows of 8 sequences from a bf16 head, the 50 likeliest tokens
        _probs("probs_7b_b8_bf16", 48, 32000, dtype="bf16", temperature=0.7, top_k=50),
        # one token each of 64 requests with settings of their own (some greedy) on a vocabulary of odd size
        _probs("probs_large_mixed", 64, 128001, temperature=1.0, top_p=0.95, mixed=True),
        # verify blocks of 64 sequences, temperature alone: the most logits
        _probs("probs_b64_blocks", 576, 32000, temperature=1.0, pad=64),
        # one sequence of the tiny decoder, drafted greedily (no drafter probabilities), no bonus row
        _verify("verify_tiny_greedy", 1, 1024, 4, 4, bonus=False, greedy=True),
        # one sequence of the 7B-shaped decoder, drafts sampled from the drafter
        _verify("verify_7b", 1, 32000, 5, 5),
        # 64 sequences with 1 to 8 drafts each
        _verify("verify_b64_ragged", 64, 32000, 1, 8),
        # 128 sequences on the large vocabulary: the most probabilities
        _verify("verify_b128_large", 128, 128001, 8, 8),
        # a speculative step's pages of 8 sequences: taken for 6 rows each, given back past what was kept
        _plan("plan_b8_block", 8, 16, 128, 2048, 6, 6),
        # 64 slots take prompts of up to 1500 tokens, then each keeps what it reached
        _plan("plan_b64_prompts", 64, 16, 0, 300, 9, 1500),
        # 1024 sequences with contexts up to 16384, blocks of up to 9 rows, a quarter of them ending
        _plan("plan_b1024", 1024, 64, 40, 16384, 1, 9, ending=0.25),
    ]


def _probs(name, rows, vocab, dtype="f32", temperature=1.0, top_k=0, top_p=1.0, mixed=False, pad=0):
    return dict(name=name, op="probs", rows=rows, vocab=vocab, dtype=dtype, temperature=temperature, top_k=top_k,
                top_p=top_p, mixed=mixed, pad=pad)


def _verify(name, batch, vocab, k_lo, k_hi, bonus=True, greedy=False):
    return dict(name=name, op="verify", batch=batch, vocab=vocab, k_lo=k_lo, k_hi=k_hi, bonus=bonus, greedy=greedy)


def _plan(name, batch, page, ctx_lo, ctx_hi, rows_lo, rows_hi, ending=0.0):
    return dict(name=name, op="plan", batch=batch, page=page, ctx_lo=ctx_lo, ctx_hi=ctx_hi, rows_lo=rows_lo,
                rows_hi=rows_hi, ending=ending)


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["probs", "probs", "verify", "verify", "plan"])
    most = {c["name"]: work(c)["bytes"] for c in listed()}
    while True:
        if op == "probs":
            top_p = rng.choice([1.0, 1.0, round(rng.uniform(0.5, 0.99), 3)])
            top_k = rng.choice([0, 0, _log_int(rng, 1, 1000)])
            c = _probs("", _log_int(rng, 1, 576), _log_int(rng, 1000, 128001), rng.choice(["f32", "f32", "bf16"]),
                       round(rng.uniform(0.3, 1.5), 3), top_k, top_p, rng.random() < 0.3, rng.choice([0, 0, 1, 64]))
            fits = work(c)["bytes"] <= most["probs_b64_blocks"]
        elif op == "verify":
            k = rng.randint(1, 16)
            c = _verify("", _log_int(rng, 1, 256), _log_int(rng, 1000, 128001), rng.choice([k, rng.randint(0, k)]), k,
                        rng.random() < 0.7, rng.random() < 0.3)
            fits = (work(c)["bytes"] <= most["verify_b128_large"] and
                    c["batch"] * (c["k_hi"] + 1) * c["vocab"] <= 128 * 9 * 128001)
        else:
            hi, r = _log_int(rng, 1, 16384), _log_int(rng, 1, 2048)
            c = _plan("", _log_int(rng, 1, 1024), rng.choice([16, 32, 64, 128]), int(hi * rng.uniform(0.0, 1.0)), hi,
                      max(1, int(r * rng.uniform(0.1, 1.0))), r, rng.choice([0.0, 0.25, 1.0]))
            fits = work(c)["bytes"] <= most["plan_b64_prompts"] and c["batch"] * (hi + r) <= 1024 * (16384 + 9)
        if fits:
            del c["name"]
            return c


# ---------------------------------------------------------------- sizes


def _spread(lo, hi, n):
    return [hi - (hi - lo) * b // max(1, n - 1) for b in range(n)]


def _drafts(c):
    return _spread(c["k_lo"], c["k_hi"], c["batch"])


def _lens(c):
    """Cached tokens of each sequence before the call, the longest first; rows: the longest get the fewest."""
    return _spread(c["ctx_lo"], c["ctx_hi"], c["batch"]), _spread(c["rows_lo"], c["rows_hi"], c["batch"])[::-1]


def _ends(c):
    """Whether a sequence ends with this step."""
    return [int((b + 1) * c["ending"]) > int(b * c["ending"]) for b in range(c["batch"])]


def work(case):
    c = case
    if c["op"] == "probs":
        n = c["rows"] * c["vocab"]
        return {"bytes": float(n * (4 + (2 if c["dtype"] == "bf16" else 4))), "flops": float(n * 6)}
    if c["op"] == "verify":
        # a row of each sequence's target and (unless drafted greedily) of its drafter; a few words a draft
        n = c["batch"] * c["vocab"]
        per = sum(_drafts(c)) * (4 * 4 if not c["greedy"] else 3 * 4) + c["batch"] * 4 * (4 + c["k_hi"])
        return {"bytes": float(n * (4 if c["greedy"] else 8) + per), "flops": float(n * 3)}
    P, moved, total = c["page"], 0, 0
    lens, rows = _lens(c)
    for n, t, e in zip(lens, rows, _ends(c)):
        held, want = -(-n // P), -(-(n + t) // P)
        moved += (want - held) + (want if e else want - held)
        total += t
    # a moved page: its entry in the stack and in the table, each read or written; a row: its slot and position
    return {"bytes": float(8 * moved + 12 * total + 4 * 8 * c["batch"]), "flops": float(4 * (moved + total))}


# ---------------------------------------------------------------- inputs


def _ints(values):
    return torch.tensor(values, dtype=torch.int32).to(DEV)


def _starts(counts):
    out = [0]
    for t in counts:
        out.append(out[-1] + t)
    return out


def _logits(n, vocab, g):
    x = 2.0 * torch.randn(n, vocab, device=DEV, generator=g)
    at = torch.randint(0, vocab, (n, 12), device=DEV, generator=g)
    return x.scatter_add_(1, at, 3.0 + 7.0 * torch.rand(n, 12, device=DEV, generator=g))


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    if c["op"] == "probs":
        n, V = c["rows"], c["vocab"]
        x = _logits(n, V + c["pad"], g)[:, :V]                 # a head padded for its matrix product: rows lie apart
        s = dict(case=c, logits=x.to(torch.bfloat16) if c["dtype"] == "bf16" else x, temperature=c["temperature"],
                 top_k=c["top_k"], top_p=c["top_p"])
        if c["mixed"]:
            # every request has its own settings; an eighth of them is greedy
            t = c["temperature"] * (0.5 + torch.rand(n, device=DEV, generator=g))
            s["temperature"] = torch.where(torch.rand(n, device=DEV, generator=g) < 0.125, 0.0, t)
            s["top_p"] = 1.0 - (1.0 - c["top_p"]) * 2.0 * torch.rand(n, device=DEV, generator=g)
            k = torch.randint(1, 200, (n,), device=DEV, generator=g)
            s["top_k"] = torch.where(torch.rand(n, device=DEV, generator=g) < 0.5, 0, k).to(torch.int32)
        return s
    if c["op"] == "verify":
        B, V, K = c["batch"], c["vocab"], _drafts(c)
        extra = 1 if c["bonus"] else 0
        total = sum(K)
        # target rows of each sequence: one a draft, and the bonus row
        x = _logits(total + extra * B, V, g)
        p = torch.softmax(x, -1)
        p = torch.where(p > 1e-4 * p.amax(-1, keepdim=True), p, 0.0)         # what a nucleus leaves
        p /= p.sum(-1, keepdim=True)
        rows = [r + extra * b for b, (a, e) in enumerate(zip(_starts(K), _starts(K)[1:])) for r in range(a, e)]
        z = x[torch.tensor(rows, dtype=torch.long).to(DEV)]
        z += torch.randn(z.shape, device=DEV, generator=g)
        del x
        q = torch.softmax(z, -1)
        noise = torch.rand(q.shape, device=DEV, generator=g).clamp_min_(1e-30).log_().neg_()
        ids = (z if c["greedy"] else q / noise).argmax(-1).to(torch.int32)
        return dict(case=c, target=p, draft=None if c["greedy"] else q, ids=ids,
                    start=_ints(_starts(K)) if min(K) != max(K) else None, n_seqs=B, most=max(K), extra=extra,
                    u_accept=torch.rand(total, device=DEV, generator=g), u_token=torch.rand(B, device=DEV, generator=g))
    B, P = c["batch"], c["page"]
    lens, rows = _lens(c)
    held = [-(-n // P) for n in lens]
    want = [-(-(n + t) // P) for n, t in zip(lens, rows)]
    n_pages, width = sum(want) + 7, max(want) + 1
    order = torch.randperm(n_pages, device=DEV, generator=g).to(torch.int32)
    cols = torch.arange(width, device=DEV)
    at = _ints(_starts(held)[:-1]).long()[:, None] + cols
    table = torch.where(cols < _ints(held)[:, None], order[at.clamp_max(n_pages - 1)], -1).to(torch.int32)
    n_free = n_pages - sum(held)
    free = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    free[:n_free] = order[sum(held):]
    # what is kept of the rows: some of a block's drafts are rejected; a sequence that ends keeps nothing
    kept = _ints(lens) + (_ints(rows) * torch.rand(B, device=DEV, generator=g)).to(torch.int32)
    kept = torch.where(_ints([int(e) for e in _ends(c)]) > 0, 0, kept)
    s = dict(case=c, free=free, n_free=_ints([n_free]), table=table, held=_ints(held), lens=_ints(lens),
             rows=_ints(rows), kept=kept, n_rows=sum(rows))
    if own:
        from paper_2510_05421_gb300 import PagePool
        s["pool"] = PagePool(s["free"], s["n_free"], s["table"], s["held"], page_tokens=P)
    return s


# ---------------------------------------------------------------- one pass


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    c = s["case"]
    if c["op"] == "probs":
        from paper_2510_05421_gb300 import token_probs
        return token_probs(s["logits"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"])
    if c["op"] == "verify":
        from paper_2510_05421_gb300 import verify_drafts
        ids, n_committed, n_accepted = verify_drafts(s["target"], s["ids"], s["u_accept"], s["u_token"],
                                                     draft=s["draft"], draft_start=s["start"], max_drafts=s["most"],
                                                     bonus=c["bonus"])
        return {"ids": ids, "n_committed": n_committed, "n_accepted": n_accepted}
    plan = s["pool"].plan(s["lens"], s["rows"], n_rows=s["n_rows"])
    s["pool"].trim(s["kept"])
    return {"row_start": plan.row_start, "slots": plan.slots, "positions": plan.positions, "table": s["table"],
            "held": s["held"], "free": s["free"], "n_free": s["n_free"]}


def _column(v, like):
    """A setting of all rows or one for each, as a column."""
    return v[:, None].to(like) if isinstance(v, torch.Tensor) else torch.full((1, 1), v, dtype=like, device=DEV)


def _run_plain(s):
    c = s["case"]
    if c["op"] == "probs":
        return _plain_probs(s)
    if c["op"] == "verify":
        return _plain_verify(s)
    got = _plain_plan(s, s["lens"], s["rows"], s["n_rows"])
    _plain_plan(s, s["kept"], torch.zeros_like(s["rows"]), 0)
    return dict(got, table=s["table"], held=s["held"], free=s["free"], n_free=s["n_free"])


def _plain_probs(s):
    c = s["case"]
    x = s["logits"].float()
    V = x.shape[1]
    T = _column(s["temperature"], torch.float32)
    top = x.amax(-1, keepdim=True)
    w = torch.exp((x - top) / torch.where(T > 0, T, 1.0))
    if c["mixed"] or c["top_k"] or c["top_p"] < 1.0:
        # in order of the logits (equal ones by index); which tokens stay is decided in 64 bits
        xs, at = x.sort(dim=-1, descending=True, stable=True)
        k, p = _column(s["top_k"], torch.int64), _column(s["top_p"], torch.float32).double()
        ws = torch.exp((xs - top).double() / torch.where(T > 0, T, 1.0).double())
        ws = torch.where((torch.arange(V, device=DEV) < k) | (k == 0), ws, 0.0)
        before = ws.cumsum(-1) - ws
        stay = (ws > 0) & ((before < p * ws.sum(-1, keepdim=True)) | (p >= 1.0))
        w = torch.where(torch.zeros_like(stay).scatter_(1, at, stay), w, 0.0)
    w = w / w.sum(-1, keepdim=True, dtype=torch.float64).float()
    if c["mixed"]:
        greedy = torch.arange(V, device=DEV) == x.argmax(-1, keepdim=True)
        w = torch.where(T > 0, w, greedy.float())
    return w


def _plain_verify(s):
    c = s["case"]
    B, K, extra = s["n_seqs"], s["most"], s["extra"]
    ids, p = s["ids"].long(), s["target"]
    start = s["start"].long() if s["start"] is not None else torch.arange(B + 1, device=DEV) * (ids.numel() // B)
    n = start.diff()
    j = torch.arange(K, device=DEV)
    has = j < n[:, None]
    at = torch.where(has, start[:-1, None] + j, 0)                         # [B, K] rows of the drafts
    row = torch.arange(B, device=DEV)[:, None] * extra + at                # and of the target
    x = ids[at]
    px = p[row, x].double()
    qx = s["draft"][at, x].double() if s["draft"] is not None else torch.ones_like(px)
    accept = has & (s["u_accept"][at].double() * qx < px)
    m = accept.int().cumprod(1).sum(1)
    # the first rejected draft's row (what the target has over the drafter), or the bonus row
    rejected = m < n
    first = start[:-1] + torch.arange(B, device=DEV) * extra
    pr = p[(first + m).clamp_max(p.shape[0] - 1)].double()
    dr = (start[:-1] + m).clamp_max(max(ids.numel() - 1, 0))
    if s["draft"] is not None:
        qr = s["draft"][dr].double()
    else:
        qr = (torch.arange(p.shape[1], device=DEV) == ids[dr][:, None]).double()
    r = torch.where(rejected[:, None], (pr - qr).clamp_min(0.0), pr)
    r = torch.where(r.sum(-1, keepdim=True) > 0, r, pr)
    cum = r.cumsum(-1)
    tok = (cum > s["u_token"].double()[:, None] * cum[:, -1:]).int().argmax(-1)
    some = rejected | (extra == 1)
    out = torch.cat([x, x.new_zeros(B, extra)], 1)
    col = torch.arange(K + extra, device=DEV)
    out = torch.where(col < m[:, None], out, torch.where((col == m[:, None]) & some[:, None], tok[:, None], -1))
    return {"ids": out.to(torch.int32), "n_committed": (m + some).to(torch.int32), "n_accepted": m.to(torch.int32)}


def _plain_plan(s, lens, rows, n_rows):
    P = s["case"]["page"]
    table, free, held = s["table"], s["free"], s["held"].long()
    n_pages, cols = free.numel(), torch.arange(table.shape[1], device=DEV)
    lens, rows = lens.long(), rows.long()
    want = (lens + rows + P - 1) // P
    # pages past what is wanted go onto the stack, in order of the sequences
    back = (held - want).clamp_min(0)
    to = s["n_free"].long() + back.cumsum(0) - back
    gives = (cols >= want[:, None]) & (cols < held[:, None])
    stack = torch.cat([free, free.new_zeros(1)])
    stack.scatter_(0, torch.where(gives, to[:, None] + cols - want[:, None], n_pages).view(-1), table.view(-1))
    n_free = s["n_free"].long() + back.sum()
    # and what is wanted past the held ones comes off its top
    new = (want - held).clamp_min(0)
    frm = n_free - 1 - (new.cumsum(0) - new)
    takes = (cols >= held[:, None]) & (cols < want[:, None])
    page = stack[torch.where(takes, frm[:, None] - (cols - held[:, None]), n_pages)]
    table.copy_(torch.where(takes, page, torch.where(cols < want[:, None], table, -1)))
    free.copy_(stack[:-1])
    s["held"].copy_(want)
    s["n_free"].copy_(n_free - new.sum())
    row_start = torch.cat([rows.new_zeros(1), rows.cumsum(0)])
    r = torch.arange(n_rows, device=DEV)
    b = torch.searchsorted(row_start[1:].contiguous(), r, right=True)
    pos = lens[b] + r - row_start[b]
    slots = table[b, pos // P].long() * P + pos % P
    return {"row_start": row_start.to(torch.int32), "slots": slots, "positions": pos.to(torch.int32)}


# ---------------------------------------------------------------- the definition in 64 bits


def exact(case, seed):
    s = prepare(dict(case), seed)
    if case["op"] == "probs":
        return _exact_probs(s)
    if case["op"] == "verify":
        return _exact_verify(s)
    return _exact_plan(s)


def _exact_probs(s):
    n, V = s["logits"].shape

    def each(v):
        return v.tolist() if isinstance(v, torch.Tensor) else [v] * n

    out = torch.zeros(n, V, dtype=torch.float64, device=DEV)
    for r, (T, k, p) in enumerate(zip(each(s["temperature"]), each(s["top_k"]), each(s["top_p"]))):
        x = s["logits"][r].double()
        if T == 0.0:
            out[r, (x == x.max()).nonzero()[0]] = 1.0
            continue
        # a setting given as a number reaches the operator as f32
        T, p = (torch.tensor(v, dtype=torch.float32).item() for v in (T, p))
        full = torch.softmax(x / T, 0)
        left = torch.argsort(-x, stable=True)[:k or V]
        if p < 1.0:
            f = full[left] / full[left].sum()
            left = left[:1 + int((f.cumsum(0) < p).sum())]
        out[r, left] = full[left] / full[left].sum()
    return out


def _exact_verify(s):
    c = s["case"]
    K, extra, width = _drafts(c), s["extra"], s["most"] + s["extra"]
    ids, ua, ut = s["ids"].tolist(), s["u_accept"].tolist(), s["u_token"].tolist()
    out, committed, accepted, a = [], [], [], 0
    for b, k in enumerate(K):
        got, m = [], 0
        while m < k:
            t, row = ids[a + m], a + m + extra * b
            q = 1.0 if s["draft"] is None else float(s["draft"][a + m, t])
            if not ua[a + m] * q < float(s["target"][row, t]):
                break
            got.append(t)
            m += 1
        accepted.append(m)
        if m < k or extra:
            p = s["target"][a + m + extra * b].double().cpu()
            r = p.clone()
            if m < k and s["draft"] is not None:
                r = (p - s["draft"][a + m].double().cpu()).clamp(min=0)
            elif m < k:
                r[ids[a + m]] = max(0.0, float(p[ids[a + m]]) - 1.0)
            if float(r.sum()) == 0.0:
                r = p
            cum = r.cumsum(0)
            got.append(int(torch.searchsorted(cum, ut[b] * float(cum[-1]), right=True)))
        committed.append(len(got))
        out.append(got + [-1] * (width - len(got)))
        a += k
    return {"ids": torch.tensor(out, dtype=torch.int32), "n_committed": torch.tensor(committed, dtype=torch.int32),
            "n_accepted": torch.tensor(accepted, dtype=torch.int32)}


def _exact_plan(s):
    P = s["case"]["page"]
    stack = s["free"].tolist()
    top = int(s["n_free"])
    width = s["table"].shape[1]
    tables = [t[:h] for t, h in zip(s["table"].tolist(), s["held"].tolist())]

    def move(lens, rows):
        nonlocal top
        want = [-(-(n + t) // P) for n, t in zip(lens, rows)]
        for t, w in zip(tables, want):
            for page in t[w:]:
                stack[top] = page
                top += 1
            del t[w:]
        for t, w in zip(tables, want):
            while len(t) < w:
                top -= 1
                t.append(stack[top])

    lens, rows = s["lens"].tolist(), s["rows"].tolist()
    move(lens, rows)
    pos = [n + i for n, t in zip(lens, rows) for i in range(t)]
    slots = [tables[b][(lens[b] + i) // P] * P + (lens[b] + i) % P for b, t in enumerate(rows) for i in range(t)]
    move(s["kept"].tolist(), [0] * len(lens))
    full = [t + [-1] * (width - len(t)) for t in tables]
    return {"row_start": torch.tensor(_starts(rows), dtype=torch.int32), "slots": torch.tensor(slots, dtype=torch.int64),
            "positions": torch.tensor(pos, dtype=torch.int32), "table": torch.tensor(full, dtype=torch.int32),
            "held": torch.tensor([len(t) for t in tables], dtype=torch.int32),
            "free": torch.tensor(stack, dtype=torch.int32), "n_free": torch.tensor([top], dtype=torch.int32)}
