"""The paged cache's operators in 64 bits, row by row (NumPy), for the tests."""
import numpy as np

TOP = {"int8": 127.0, "e4m3": 448.0}
MIN_SCALE = 2.0 ** -80


def e4m3_values():
    """The 256 values of the e4m3 byte codes (NaN at 0x7f and 0xff)."""
    out = np.empty(256)
    for c in range(256):
        e, f = (c >> 3) & 15, c & 7
        v = np.nan if e == 15 and f == 7 else (f / 8 * 2.0 ** -6 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7))
        out[c] = -v if c & 128 else v
    return out


E4M3 = e4m3_values()


def values(codes, fmt):
    return codes.astype(np.float64) if fmt == "int8" else E4M3[codes.view(np.uint8)]


def step_of(code_value, fmt):
    """Distance between neighbouring codes at a value (in units of the scale)."""
    if fmt == "int8":
        return np.ones_like(code_value)
    a = np.maximum(np.abs(code_value), 2.0 ** -6)
    return 2.0 ** (np.floor(np.log2(a)) - 3)


def rotate(x, pos, rotary):
    """x [H, D] at position pos; rotary [n_pos, rot / 2, 2]."""
    if rotary is None or pos >= rotary.shape[0]:
        return x
    h = rotary.shape[1]
    c, s = rotary[pos, :, 0].astype(np.float64), rotary[pos, :, 1].astype(np.float64)
    y = x.copy()
    y[:, :h] = x[:, :h] * c - x[:, h:2 * h] * s
    y[:, h:2 * h] = x[:, h:2 * h] * c + x[:, :h] * s
    return y


def attend(kv, table, lens, starts, q, scale, softcap=0.0, window=0, slopes=None):
    """kv: dict of codes k, v [n_pages, H, P, D], k_scale, v_scale [n_pages, H], fmt.  Returns (o, bound per
    row and head: sum of p |v| per dim, largest sum |q k| scale) for tolerances."""
    fmt = kv["fmt"]
    n_pages, H, P, D = kv["k"].shape
    K = values(kv["k"], fmt) * kv["k_scale"].astype(np.float64)[:, :, None, None]
    V = values(kv["v"], fmt) * kv["v_scale"].astype(np.float64)[:, :, None, None]
    n, Hq, _ = q.shape
    o, mass, reach = np.zeros((n, Hq, D)), np.zeros((n, Hq, D)), np.zeros((n, Hq))
    for b in range(len(lens)):
        for r in range(starts[b], starts[b + 1]):
            p = int(lens[b]) + r - starts[b]
            keys = [j for j in range(max(0, p - window + 1) if window else 0, p + 1)
                    if j // P < table.shape[1] and table[b, j // P] >= 0]
            if not keys:
                continue
            j = np.array(keys)
            pg = table[b, j // P]
            for h in range(Hq):
                kh, vh = K[pg, h * H // Hq, j % P], V[pg, h * H // Hq, j % P]
                s = kh @ q[r, h] * scale
                reach[r, h] = (np.abs(kh) @ np.abs(q[r, h])).max() * scale
                if softcap:
                    s = softcap * np.tanh(s / softcap)
                if slopes is not None:
                    s = s + float(slopes[h]) * (j - p)
                    reach[r, h] += abs(float(slopes[h])) * len(range(j[0], p + 1))
                w = np.exp(s - s.max())
                w /= w.sum()
                o[r, h] = w @ vh
                mass[r, h] = w @ np.abs(vh)
    return o, mass, reach


def attend_bound(o, mass, reach, keys, head_dim, dtype, largest=0.0):
    """How far an attention result may be from `attend`'s, of rows that see up to `keys` positions: a score is off by
    at most reach (head_dim + 8) 2^-23 (f32 products and sums that may truncate), which moves the result by twice that
    times the mass; a weight's f16 rounding is 2^-11 of it (f32 queries: two f16 numbers, 2^-21), the sums of the
    weights (keys / 16 + 64) 2^-23 of the mass, and a bf16 result is rounded by 2^-8 of itself.  Where the weights of a
    row spread past f16's range, those far below its largest (at least 2^5 in f16) are off by up to 2^-25: with `largest`,
    the largest |v|, that counts too."""
    tol = mass * (2 * reach[..., None] * (head_dim + 8) * 2.0 ** -23 + (keys / 16 + 64) * 2.0 ** -23 +
                  (2.0 ** -11 if dtype == "bf16" else 2.0 ** -21)) + keys * 2.0 ** -30 * largest + 1e-30
    return tol + np.abs(o) * 2.0 ** -8 if dtype == "bf16" else tol
