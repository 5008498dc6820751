"""verify_drafts with starts that fall or lie outside the drafts: cut to them as the header says, every output as the
definition gives it for the cut starts, and nothing read around the arrays.

Every array lies within a larger one that is filled with what would show: NaN (flagged), ids of the vocabulary (which
would be accepted or rejected otherwise).  The starts are a few entries off, so a mistaken read stays inside."""
import numpy as np
import pytest
import torch

from sampling_ref import verify
from test_gpu_verify_drafts import case

pytestmark = pytest.mark.gpu

AROUND = 16


def within(a, fill):
    """`a` on the GPU with AROUND rows of `fill` before and behind it."""
    a = torch.from_numpy(np.ascontiguousarray(a))
    big = torch.full((len(a) + 2 * AROUND, *a.shape[1:]), fill, dtype=a.dtype)
    big[AROUND:AROUND + len(a)] = a
    return big.cuda()[AROUND:AROUND + len(a)]


def definition(p, ids, ua, ut, q, start, bonus, most):
    """Sequence by sequence, on the rows that its cut starts name."""
    n, out, nc, na = len(ids), [], [], []
    for b in range(len(ut)):
        lo = min(max(start[b], 0), n)
        hi = min(max(start[b + 1], lo), n)
        k = min(hi - lo, most)
        at = slice(lo, lo + k)
        row = lo + b * bonus
        got = verify(p[row:row + k + bonus], ids[at], ua[at], ut[b:b + 1], None if q is None else q[at], [k], bonus, most)
        for to, x in zip((out, nc, na), got):
            to.append(x[0])
    return np.array(out).reshape(len(ut), most + bonus), np.array(nc), np.array(na)


@pytest.mark.parametrize("start", [[0, 9, 4, 6], [-3, 2, 4, 6], [0, 2, 4, 9], [3, 1, -2, 8], [6, 5, 4, 3], [2, 2, 2, 2],
                                   [9, 9, 9, 9], [-5, -4, -3, -2], [0, 6, 0, 6], [0, -1, 7, 2]])
@pytest.mark.parametrize("bonus", [False, True])
@pytest.mark.parametrize("greedy", [False, True])
def test_starts(start, bonus, greedy):
    from paper_2510_05421_gb300 import verify_drafts
    p, ids, ua, ut, q = case([2, 2, 2], 300, 9, int(bonus), greedy)
    p = np.maximum(p, np.float32(1e-6))
    cut = [min(max(x, 0), 6) for x in start]
    flag = 8 if any(a != b for a, b in zip(start, cut)) or cut != sorted(cut) else 0
    for share, most in ((1.0, 6), (1.0, 1), (0.0, 6), (0.0, 2)):      # (a share of 0: all drafts are accepted)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        got = verify_drafts(within(p, torch.nan), within(ids, 7), within(ua * np.float32(share), 0.0), within(ut, torch.nan),
                            draft=None if greedy else within(q, torch.nan), draft_start=within(np.array(start, np.int32), 3),
                            max_drafts=most, bonus=bonus, status=status)
        torch.cuda.synchronize()
        for a, b in zip(got, definition(p, ids, ua * np.float32(share), ut, q, start, int(bonus), most)):
            np.testing.assert_array_equal(a.cpu().numpy(), b)
        assert int(status) == flag
