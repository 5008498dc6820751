"""The 8-bit paged KV cache's operators as measurable cases: append, attend, read.

A program that serves many sequences with this library keeps keys and values
in pages of 8-bit codes with an f32 scale for each page and KV head.  Each
decoder pass appends the rows of its new tokens (one for a draft pass or a
greedy step, K or K + 1 for a verify block, hundreds for a prompt chunk;
ragged across the batch), attends to everything cached, and now and then reads
cached rows back as values (to move a sequence or to hand it to a 16-bit
path).  The listed cases use the repository's decoders (tiny: 4 heads of 64;
mid: 16 over 4; 1B-shaped: 16 over 8 of 128; 7B-shaped: 32 of 128) with
contexts of 64 to 16384 tokens; draw() spreads more over the same ranges, with
other head groups, page sizes, odd lengths and ragged batches.

Keys and queries are normal draws with scores of standard deviation 2, pages
lie in random order, and the rows of a last page that no token fills yet hold
an earlier request's codes.
"""
from __future__ import annotations

import math

import torch

own = False      # True: the library's operators; False: the same in elementary torch operations

DEV = "cuda"
CODE_MAX = {"int8": 127.0, "e4m3": 448.0}
MIN_SCALE = 2.0 ** -80


def _case(op, heads, kv_heads, head_dim, **kw):
    c = dict(op=op, heads=heads, kv_heads=kv_heads, head_dim=head_dim, dtype="bf16", fmt="int8", page=64, batch=1,
             ctx_lo=0, ctx_hi=0, rows_lo=1, rows_hi=1, softcap=0.0, window=0, slopes=False)
    c.update(kw)
    return c


def _named(name, c):
    return dict(c, name=name)


def listed():
    return [
        # one greedy token of the 1B-shaped decoder enters a page that has rows: the smallest append
        _named("append_1b_token", _case("append", 16, 8, 128, ctx_lo=540, ctx_hi=540)),
        # a ragged batch of prompt chunks on the 7B-shaped decoder, pages of 16
        _named("append_7b_prompts", _case("append", 32, 32, 128, fmt="e4m3", page=16, batch=8, ctx_lo=0, ctx_hi=99,
                                          rows_lo=128, rows_hi=2048)),
        # the last 64 tokens of one sequence back as values
        _named("read_1b_64", _case("read", 16, 8, 128, ctx_lo=448, ctx_hi=448, rows_lo=64, rows_hi=64)),
        # a whole 16384-token sequence of the 7B-shaped decoder back as values
        _named("read_7b_16k", _case("read", 32, 32, 128, fmt="e4m3", rows_lo=16384, rows_hi=16384)),
        # one greedy token of the 1B-shaped decoder over a chat-sized context: latency counts
        _named("attend_1b_token", _case("attend", 16, 8, 128, ctx_lo=540, ctx_hi=540)),
        # the tiny f32 decoder's verify block, with a distance bias
        _named("attend_tiny_f32", _case("attend", 4, 4, 64, dtype="f32", page=16, ctx_lo=75, ctx_hi=75, rows_lo=5,
                                        rows_hi=5, slopes=True)),
        # greedy tokens of a ragged batch of 8 on the 7B-shaped decoder, pages of 16
        _named("attend_7b_b8", _case("attend", 32, 32, 128, fmt="e4m3", page=16, batch=8, ctx_lo=128, ctx_hi=2560)),
        # the verify block of 9 rows over 16384 cached positions
        _named("attend_7b_16k", _case("attend", 32, 32, 128, ctx_lo=16384, ctx_hi=16384, rows_lo=9, rows_hi=9)),
        # 64 sequences of a mid-sized decoder, capped scores and a sliding window
        _named("attend_mid_b64", _case("attend", 16, 4, 64, fmt="e4m3", page=32, batch=64, ctx_lo=100, ctx_hi=8192,
                                       softcap=30.0, window=4096)),
        # verify blocks of 32 long sequences: the most cache
        _named("attend_1b_b32_16k", _case("attend", 16, 8, 128, batch=32, ctx_lo=12000, ctx_hi=16384, rows_lo=6,
                                          rows_hi=6)),
        # a ragged batch of short prompts from empty caches
        _named("attend_1b_prompts", _case("attend", 16, 8, 128, batch=8, rows_lo=23, rows_hi=301)),
        # a long prompt's chunk behind what is cached: the most arithmetic
        _named("attend_7b_chunk", _case("attend", 32, 32, 128, ctx_lo=3001, ctx_hi=3001, rows_lo=1000, rows_hi=1000)),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        c = _draw(rng)
        ctx, rows = _lens(c), _rows(c)
        room = max(n + t for n, t in zip(ctx, rows))
        held = c["batch"] * room * c["kv_heads"] * c["head_dim"]          # codes of K, padded to the longest
        scores = c["batch"] * max(rows) * c["heads"] * room if c["op"] == "attend" else 0
        moved = sum(rows) * (c["heads"] + 2 * c["kv_heads"]) * c["head_dim"] if c["op"] != "attend" else 0
        if held <= 32 * 16390 * 8 * 128 and scores <= 32 * 1000 * 4001 and moved <= 16384 * 64 * 128:
            w = work(c)
            if w["bytes"] <= work(_most_bytes())["bytes"] and w["flops"] <= work(_most_flops())["flops"]:
                return c


def _most_bytes():
    return max(listed(), key=lambda c: work(c)["bytes"])


def _most_flops():
    return max(listed(), key=lambda c: work(c)["flops"])


def _draw(rng):
    op = rng.choice(["append", "append", "read", "attend", "attend", "attend", "attend"])
    kv = rng.choice([1, 2, 4, 8, 8, 32])
    group = rng.choice([1, 1, 2, 3, 4, 4, 7, 8] if kv < 32 else [1])
    batch = _log_int(rng, 1, 64)
    hi = _log_int(rng, 1, 16384)
    kind = rng.choice(["token", "block", "prompt"])
    r_hi = {"token": 1, "block": rng.randint(2, 17), "prompt": _log_int(rng, 18, 2048)}[kind]
    if op == "read":
        r_hi = _log_int(rng, 1, 16384)
    c = _case(op, kv * group, kv, rng.choice([64, 128]), dtype=rng.choice(["bf16"] * 4 + ["f32"]),
              fmt=rng.choice(["int8", "e4m3"]), page=rng.choice([16, 32, 64, 128]), batch=batch,
              ctx_lo=int(hi * rng.uniform(0.1, 1.0)), ctx_hi=hi,
              rows_lo=r_hi if rng.random() < 0.5 else max(1, int(r_hi * rng.uniform(0.2, 1.0))), rows_hi=r_hi)
    if op == "attend":
        c["softcap"] = rng.choice([0.0, 0.0, 0.0, 30.0, 50.0])
        c["window"] = rng.choice([0, 0, 0, _log_int(rng, 64, 8192)])
        c["slopes"] = rng.random() < 0.25
    return c


# ---------------------------------------------------------------- sizes


def _spread(lo, hi, n):
    return [hi - (hi - lo) * b // max(1, n - 1) for b in range(n)]


def _lens(c):
    """Cached tokens of each sequence before the call, the longest first."""
    return _spread(c["ctx_lo"], c["ctx_hi"], c["batch"])


def _rows(c):
    """New rows of each sequence: the longest contexts get the fewest."""
    return _spread(c["rows_lo"], c["rows_hi"], c["batch"])[::-1]


def work(case):
    c = case
    H, Hq, D, e = c["kv_heads"], c["heads"], c["head_dim"], 4 if c["dtype"] == "f32" else 2
    rows, lens = _rows(c), _lens(c)
    n = sum(rows)
    if c["op"] == "append":
        # the rows in, the codes and the rotated queries out; then the touched pages read back as values
        back = sum(x for _, x in _touched(c))
        return {"bytes": float(n * D * (e * (2 * H + 2 * Hq) + 2 * H + 4) + back * 2 * H * D * (1 + e)),
                "flops": float(n * D * 3 * (2 * H + Hq))}
    if c["op"] == "read":
        return {"bytes": float(n * 2 * H * D * (1 + e)), "flops": float(2 * n * H * D)}
    seen = pairs = 0
    for n0, t in zip(lens, rows):
        w = c["window"] or (n0 + t)
        seen += n0 + t - max(0, n0 + 1 - w)
        # row i sees min(n0 + i + 1, w) positions
        full = max(0, min(t, w - n0 - 1))
        pairs += full * (2 * n0 + full + 1) // 2 + (t - full) * w
    return {"bytes": float(seen * 2 * H * D + 2 * n * Hq * D * e), "flops": float(4 * D * Hq * pairs)}


def _touched(c):
    """For each sequence the first position of the pages that the rows touch, and the positions from there on."""
    P = c["page"]
    return [(n0 // P * P, n0 + t - n0 // P * P) for n0, t in zip(_lens(c), _rows(c))]


# ---------------------------------------------------------------- inputs


def _codes(c, shape, g):
    x = torch.empty(shape, dtype=torch.bfloat16, device=DEV).normal_(0.0, 1.0, generator=g)
    if c["fmt"] == "int8":
        return x.mul_(40.0).round_().clamp_(-127, 127).to(torch.int8)
    return x.mul_(120.0).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32).to(DEV)


def _starts(rows):
    out = [0]
    for t in rows:
        out.append(out[-1] + t)
    return out


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    H, Hq, D, P, B = c["kv_heads"], c["heads"], c["head_dim"], c["page"], c["batch"]
    td = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    lens, rows = _lens(c), _rows(c)
    pages = [-(-(n + t) // P) for n, t in zip(lens, rows)]
    width, total = max(pages), sum(pages)
    n_pages = total + 3
    order = torch.randperm(n_pages, device=DEV, generator=g).to(torch.int32)
    starts = _ints(_starts(pages))
    cols = torch.arange(width, device=DEV, dtype=torch.int32)
    at = starts[:-1, None] + cols
    table = torch.where(cols < _ints(pages)[:, None], order[at.clamp_max(n_pages - 1).long()], 0).to(torch.int32)
    unit = 1.0 / (40.0 if c["fmt"] == "int8" else 120.0)
    s = dict(case=c, dtype=td, lens=_ints(lens), table=table.contiguous(), max_rows=max(rows), n_rows=sum(rows),
             row_start=_ints(_starts(rows)) if min(rows) != max(rows) else None,
             k=_codes(c, (n_pages, H, P, D), g), v=_codes(c, (n_pages, H, P, D), g),
             ks=unit * (0.6 + 0.8 * torch.rand(n_pages, H, device=DEV, generator=g)),
             vs=unit * (0.6 + 0.8 * torch.rand(n_pages, H, device=DEV, generator=g)))
    n = sum(rows)
    if c["op"] == "append":
        # one projection's output holds a row's queries, keys and values side by side
        qkv = torch.randn(n, Hq + 2 * H, D, device=DEV, generator=g).to(td)
        s.update(q=qkv[:, :Hq], k_new=qkv[:, Hq:Hq + H], v_new=qkv[:, Hq + H:])
        pos = torch.arange(max(a + b for a, b in zip(lens, rows)), device=DEV, dtype=torch.float64)
        inv = 10000.0 ** (-torch.arange(0, D, 2, device=DEV, dtype=torch.float64) / D)
        ang = pos[:, None] * inv
        s["rotary"] = torch.stack([ang.cos(), ang.sin()], -1).float().contiguous()
        back = _touched(c)
        s.update(back_lens=_ints([a for a, _ in back]), back_start=_ints(_starts([b for _, b in back])),
                 back_n=sum(b for _, b in back), back_max=max(b for _, b in back))
    elif c["op"] == "attend":
        s["q"] = (2.0 * torch.randn(n, Hq, D, device=DEV, generator=g)).to(td)
        s["slopes"] = (2.0 ** (-8.0 * torch.arange(1, Hq + 1, device=DEV) / Hq)).float() if c["slopes"] else None
    if own:
        from paper_2510_05421_gb300 import PagedCache
        s["cache"] = PagedCache(s["k"], s["v"], s["ks"], s["vs"], fmt=c["fmt"])
    return s


# ---------------------------------------------------------------- one pass


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    c, cache = s["case"], s["cache"]
    if c["op"] == "append":
        q = cache.append(s["table"], s["lens"], s["k_new"], s["v_new"], q=s["q"], rotary=s["rotary"],
                         row_start=s["row_start"], max_rows=s["max_rows"])
        k, v = cache.read(s["table"], s["back_lens"], s["back_n"], row_start=s["back_start"], max_rows=s["back_max"],
                          dtype=s["dtype"])
        return {"q": q, "k": k, "v": v, "k_scale": s["ks"], "v_scale": s["vs"]}
    if c["op"] == "read":
        k, v = cache.read(s["table"], s["lens"], s["n_rows"], row_start=s["row_start"], max_rows=s["max_rows"],
                          dtype=s["dtype"])
        return {"k": k, "v": v}
    return cache.attend(s["table"], s["lens"], s["q"], softcap=c["softcap"], window=c["window"], slopes=s["slopes"],
                        row_start=s["row_start"], max_rows=s["max_rows"])


def _rows_of(lens, row_start, n):
    """Sequence, index in the sequence and position of each row."""
    B = lens.numel()
    r = torch.arange(n, device=DEV)
    if row_start is None:
        seq = torch.div(r, n // B, rounding_mode="floor")
        i = r - seq * (n // B)
    else:
        seq = torch.searchsorted(row_start[1:].contiguous(), r.to(torch.int32), right=True)
        i = r - row_start[seq]
    return seq, i, lens[seq].long() + i


def _val(codes, fmt):
    return codes.float() if fmt == "int8" else codes.view(torch.float8_e4m3fn).float()


def _enc(x, fmt):
    top = CODE_MAX[fmt]
    if fmt == "int8":
        return x.round().clamp(-top, top).to(torch.int8)
    return x.clamp(-top, top).to(torch.float8_e4m3fn).view(torch.uint8)


def _rotate(x, cs):
    h = x.shape[-1] // 2
    a, b = x[..., :h], x[..., h:]
    cos, sin = cs[:, None, :, 0], cs[:, None, :, 1]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _store(pool, scale, x, page, off, page0, held, fmt):
    top = CODE_MAX[fmt]
    most = torch.zeros_like(scale).index_reduce_(0, page, x.abs().amax(-1), "amax")
    new = (most / top).clamp_min(MIN_SCALE)
    old = scale[page0]
    first = torch.where(held[:, None] > 0, torch.maximum(new[page0], old), new[page0])
    factor = (old / first)[:, :, None, None]
    codes = pool[page0]
    keep = torch.arange(pool.shape[2], device=DEV)[None, None, :, None] < held[:, None, None, None]
    grown = keep & (factor < 1)
    pool[page0] = torch.where(grown, _enc(_val(codes, fmt) * factor, fmt), codes)
    new[page0] = first
    scale[page] = new[page]
    pool[page, :, off] = _enc(x * (1.0 / scale[page])[..., None], fmt)


def _plain_read(s, lens, row_start, n):
    c, P = s["case"], s["case"]["page"]
    seq, _, pos = _rows_of(lens, row_start, n)
    page = s["table"][seq, pos // P].long()
    off = pos % P
    k = _val(s["k"][page, :, off], c["fmt"]) * s["ks"][page][..., None]
    v = _val(s["v"][page, :, off], c["fmt"]) * s["vs"][page][..., None]
    return k.to(s["dtype"]), v.to(s["dtype"])


def _run_plain(s):
    c = s["case"]
    P, fmt = c["page"], c["fmt"]
    if c["op"] == "read":
        k, v = _plain_read(s, s["lens"], s["row_start"], s["n_rows"])
        return {"k": k, "v": v}
    seq, i, pos = _rows_of(s["lens"], s["row_start"], s["n_rows"])
    if c["op"] == "append":
        page = s["table"][seq, pos // P].long()
        off = pos % P
        lens = s["lens"].long()
        page0 = s["table"].gather(1, (lens // P)[:, None]).squeeze(1).long()
        cs = s["rotary"][pos]
        _store(s["k"], s["ks"], _rotate(s["k_new"].float(), cs), page, off, page0, lens % P, fmt)
        _store(s["v"], s["vs"], s["v_new"].float(), page, off, page0, lens % P, fmt)
        k, v = _plain_read(s, s["back_lens"], s["back_start"], s["back_n"])
        return {"q": _rotate(s["q"].float(), cs).to(s["dtype"]), "k": k, "v": v, "k_scale": s["ks"],
                "v_scale": s["vs"]}
    B, H, Hq, D, T = c["batch"], c["kv_heads"], c["heads"], c["head_dim"], s["max_rows"]
    G, L = Hq // H, s["table"].shape[1] * P
    tab = s["table"].long()

    def dense(codes, scale):
        x = _val(codes[tab], fmt) * scale[tab][..., None, None]            # [B, pages, H, P, D]
        return x.permute(0, 2, 1, 3, 4).reshape(B, H, L, D)

    q = torch.zeros(B, T, Hq, D, device=DEV)
    q[seq, i] = s["q"].float()
    q = q.view(B, T, H, G, D).permute(0, 2, 1, 3, 4).reshape(B, H, T * G, D)
    x = torch.matmul(q, dense(s["k"], s["ks"]).transpose(2, 3)).mul_(D ** -0.5).view(B, H, T, G, L)
    if c["softcap"]:
        x = c["softcap"] * torch.tanh(x / c["softcap"])
    at = s["lens"].long()[:, None] + torch.arange(T, device=DEV)           # [B, T]
    dist = torch.arange(L, device=DEV) - at[:, :, None]                    # [B, T, L], <= 0 where seen
    if s["slopes"] is not None:
        x = x + s["slopes"].view(H, 1, G, 1) * dist[:, None, :, None, :].float()
    seen = dist <= 0
    if c["window"]:
        seen = seen & (dist > -c["window"])
    seen = seen[:, None, :, None, :]
    x = x.masked_fill(~seen, float("-inf"))
    p = torch.exp(x - x.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    held = torch.arange(L, device=DEV) <= at[:, -1:]
    v = dense(s["v"], s["vs"]).masked_fill(~held[:, None, :, None], 0.0)
    o = torch.matmul(p.view(B, H, T * G, L), v).view(B, H, T, G, D).permute(0, 2, 1, 3, 4).reshape(B, T, Hq, D)
    return o[seq, i].to(s["dtype"])


# ---------------------------------------------------------------- the definition in 64 bits


def _values64(codes, fmt):
    return (codes if fmt == "int8" else codes.view(torch.float8_e4m3fn).float()).double()


def _round64(x, fmt):
    top = CODE_MAX[fmt]
    if fmt == "int8":
        return x.round().clamp(-top, top)
    a = x.abs().clamp_max(top)
    step = torch.exp2(torch.floor(torch.log2(a.clamp_min(2.0 ** -6))) - 3)   # 3 fraction bits, from 2^-6 down fixed
    return torch.sign(x) * (a / step).round() * step


def exact(case, seed):
    c = dict(case)
    s = prepare(c, seed)
    P, fmt, D, H, Hq = c["page"], c["fmt"], c["head_dim"], c["kv_heads"], c["heads"]
    lens, rows = _lens(c), _rows(c)
    at = _starts(rows)

    def cached(codes, scale, b, n):
        """The first n positions of sequence b: [H, n, D]."""
        pg = s["table"][b, :-(-n // P)].long()
        x = _values64(codes[pg], fmt) * scale[pg].double()[..., None, None]
        return x.transpose(0, 1).reshape(H, -1, D)[:, :n]

    if c["op"] == "read":
        out = {}
        for name, codes, scale in (("k", s["k"], s["ks"]), ("v", s["v"], s["vs"])):
            out[name] = torch.cat([cached(codes, scale, b, lens[b] + rows[b])[:, lens[b]:].transpose(0, 1)
                                   for b in range(c["batch"])])
        return out
    if c["op"] == "append":
        return _exact_append(c, s, lens, rows, at)
    outs = []
    for b in range(c["batch"]):
        n, t = lens[b] + rows[b], rows[b]
        k, v = cached(s["k"], s["ks"], b, n), cached(s["v"], s["vs"], b, n)
        q = s["q"][at[b]:at[b + 1]].double()
        o = torch.empty(t, Hq, D, dtype=torch.float64, device=DEV)
        d = torch.arange(n, device=DEV)[None] - (lens[b] + torch.arange(t, device=DEV))[:, None]
        hidden = (d > 0) | ((d <= -c["window"]) if c["window"] else torch.zeros_like(d, dtype=torch.bool))
        for h in range(Hq):
            x = q[:, h] @ k[h * H // Hq].T / math.sqrt(D)
            if c["softcap"]:
                x = c["softcap"] * torch.tanh(x / c["softcap"])
            if s["slopes"] is not None:
                x = x + s["slopes"][h].double() * d
            o[:, h] = torch.softmax(x.masked_fill(hidden, -math.inf), -1) @ v[h * H // Hq]
        outs.append(o)
    return torch.cat(outs)


def _exact_append(c, s, lens, rows, at):
    P, fmt, D = c["page"], c["fmt"], c["head_dim"]
    top = CODE_MAX[fmt]
    h = D // 2

    def rot(x, b):
        cs = s["rotary"][lens[b]:lens[b] + rows[b]].double()[:, None]
        z = torch.complex(x[..., :h], x[..., h:]) * torch.complex(cs[..., 0], cs[..., 1])
        return torch.cat([z.real, z.imag], -1)

    qs, ks, vs = [], [], []
    scales = [s["ks"].double(), s["vs"].double()]
    for b in range(c["batch"]):
        part = slice(at[b], at[b + 1])
        qs.append(rot(s["q"][part].double(), b))
        fresh = (rot(s["k_new"][part].double(), b), s["v_new"][part].double())
        first = lens[b] // P
        for x, codes, scale, out in zip(fresh, (s["k"], s["v"]), scales, (ks, vs)):
            done = 0
            while done < rows[b]:
                p = lens[b] + done
                pg, held = int(s["table"][b, p // P]), p % P
                m = min(P - held, rows[b] - done)
                new = x[done:done + m].transpose(0, 1)                         # [H, m, D]
                sc = (new.abs().amax((1, 2)) / top).clamp_min(MIN_SCALE)
                if held:
                    was = scale[pg].clone()
                    sc = torch.maximum(sc, was)
                    old = _values64(codes[pg][:, :held], fmt)
                    moved = _round64(old * (was / sc)[:, None, None], fmt)
                    old = torch.where((sc > was)[:, None, None], moved, old)
                    out.append((old * sc[:, None, None]).transpose(0, 1))
                out.append((_round64(new / sc[:, None, None], fmt) * sc[:, None, None]).transpose(0, 1))
                scale[pg] = sc
                done += m
            assert first * P <= lens[b]
    return {"q": torch.cat(qs), "k": torch.cat(ks), "v": torch.cat(vs), "k_scale": scales[0], "v_scale": scales[1]}
