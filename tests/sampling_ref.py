"""Token probabilities, draft verification and page plans from their definitions, in 64 bits (NumPy), for the tests."""
import numpy as np

F32_MAX = float(np.finfo(np.float32).max)


def probs(x, T, k, p):
    """Row x (f64 values of the logits).  Returns (probabilities, tolerance of each, the smallest distance of a top-p
    decision from its border, over the row's sum; inf where there is none).

    The tolerance: exp2 of an argument t is off by 2 units (2^-22), t by three roundings of 2^-24 of itself, which moves
    the result by ln 2 times that; the normaliser and the product by three more roundings."""
    x = np.where(np.isnan(x), -np.inf, np.minimum(x, F32_MAX)).astype(np.float64)
    V = len(x)
    out = np.zeros(V)
    if np.max(x) == -np.inf:
        return out, np.zeros(V), np.inf
    if not T > 0:
        out[int(np.argmax(x))] = 1.0
        return out, np.zeros(V), np.inf
    T = min(max(float(T), 2.0 ** -100), 2.0 ** 100)
    with np.errstate(over="ignore", under="ignore"):
        t = (x - x.max()) / T
        w = np.where(x == -np.inf, 0.0, np.exp(t))
    order = np.argsort(-x, kind="stable")
    order = order[x[order] > -np.inf]
    if 0 < k < V:
        order = order[:k]
    border = np.inf
    if p < 1:
        before = np.cumsum(w[order]) - w[order]
        at = p * w[order].sum()
        keep = before < at
        keep[0] = True
        border = np.abs(before[1:] - at).min() / w[order].sum() if len(order) > 1 else np.inf
        order = order[keep]
    out[order] = w[order] / w[order].sum()
    tol = out * (np.abs(np.maximum(t, -200.0)) * 3 * 2.0 ** -24 + 2.0 ** -21) + 2.0 ** -140
    return out, np.where(out > 0, tol, 0.0), border


def verify(target, ids, ua, ut, draft, counts, bonus, most=None):
    """Returns (ids, n_committed, n_accepted) as int arrays; counts: drafts of each sequence."""
    def clean(r):
        r = r.astype(np.float64)
        return np.where(np.isfinite(r), np.maximum(r, 0.0), 0.0)

    most = max([*counts, 0]) if most is None else most
    V = target.shape[1]
    out = np.full((len(counts), most + bonus), -1, np.int64)
    nc, na, a = [], [], 0
    for b, n in enumerate(counts):
        k, m = min(n, most), 0
        while m < k:
            t = int(ids[a + m])
            if not 0 <= t < V:
                break
            q = 1.0 if draft is None else clean(draft[a + m])[t]
            if not float(ua[a + m]) * q < clean(target[a + m + b * bonus])[t]:
                break
            out[b, m] = t
            m += 1
        c = m
        if m < k or bonus:
            p = clean(target[a + m + b * bonus])
            r = p
            if m < k:
                if draft is not None:
                    q = clean(draft[a + m])
                else:
                    q = np.zeros(V)
                    if 0 <= ids[a + m] < V:
                        q[ids[a + m]] = 1.0
                r = np.maximum(p - q, 0.0)
                if r.sum() == 0:
                    r = p
            if r.sum() > 0:
                cum = np.cumsum(r)
                u = float(ut[b])
                i = int(np.searchsorted(cum, u * cum[-1], side="right")) if u >= 0 else int(np.nonzero(r)[0][0])
                out[b, m] = min(i, int(np.nonzero(r)[0][-1]))
                c += 1
        nc.append(c)
        na.append(m)
        a += n
    return out, np.array(nc), np.array(na)


class Pool:
    """A page pool as lists."""

    def __init__(self, n_pages, n_seqs, max_pages, P):
        self.stack = list(range(n_pages - 1, -1, -1))
        self.tables = [[] for _ in range(n_seqs)]
        self.max_pages, self.P = max_pages, P

    def plan(self, lens, rows):
        """Returns (row starts, slots, positions, whether a slot was passed over)."""
        lens, rows = [max(int(n), 0) for n in lens], [max(int(t), 0) for t in rows]
        want = [-(-(n + t) // self.P) for n, t in zip(lens, rows)]
        full = False
        for t, w in zip(self.tables, want):
            if w < len(t):
                self.stack += t[w:]
                del t[w:]
        for t, w in zip(self.tables, want):
            if w > self.max_pages or w - len(t) > len(self.stack):
                full = True
                continue
            while len(t) < w:
                t.append(self.stack.pop())
        start, slots, positions = [0], [], []
        for t, n, c in zip(self.tables, lens, rows):
            start.append(start[-1] + c)
            for pos in range(n, n + c):
                positions.append(pos)
                slots.append(t[pos // self.P] * self.P + pos % self.P if pos // self.P < len(t) else -1)
        return start, slots, positions, full

    def table(self):
        return np.array([t + [-1] * (self.max_pages - len(t)) for t in self.tables])
