"""How far the probabilities of tokens far below the maximum are off: by the rounding of (x - max) / T to 32 bits, which
goes either way, and not by that of 1 / T, which would go one way for all of them."""
import numpy as np
import pytest
import torch

from paper_2510_05421_gb300 import token_probs

pytestmark = pytest.mark.gpu


def temperature():
    """Of some numbers near log2(e), that whose log2(e) / T is the furthest from a number of 32 bits: nearly half a step,
    just above 1, so 2^-24 of itself."""
    t = np.nextafter(np.float32(1.4426), np.float32(0)) - np.arange(2000, dtype=np.float32) * np.float32(2.0 ** -23)
    c = np.log2(np.e) / t.astype(np.float64)
    off = (c.astype(np.float32).astype(np.float64) - c) / c
    assert np.abs(off).max() > 0.95 * 2.0 ** -24
    return float(t[np.abs(off).argmax()])


@pytest.mark.parametrize("vocab,top_k", [(2000, 0), (2000, 1999), (4001, 0), (32000, 0), (32000, 31999), (100003, 0),
                                         (100003, 90000)])
def test_far_tokens(vocab, top_k):
    """The maximum is 0, so x - max is exact; t = x log2(e) / T lies in -120 .. -64, where half a step is 2^-18, or
    2^-18 ln 2 of the probability.  exp2f is off by 2 units of 2^-23 at most, the sum is 1 but for 2^-47, the product and
    its factor have 2^-24 each.  The mean of n errors of a step's rounding (evenly spread) is within six of its standard
    deviations, 2^-17 ln 2 / sqrt(12 n).

    Without cuts a warp takes w to its own maximum m, and what it has by one factor to the row's: two roundings, of
    (x - m) log2(e) / T in -56 .. 0 (half a step 2^-19; x and m are multiples of 2^-17 below 128, so x - m is exact) and
    of m log2(e) / T (2^-18), two exp2f and two products more.  The factor is the same for a warp's tokens, 1024 at most,
    so the mean has as few independent errors as that leaves: sqrt(1024 / n) of one's deviation."""
    T = temperature()
    g = np.random.default_rng(vocab)
    x = g.uniform(-110, -64, vocab).astype(np.float32)
    x[g.integers(vocab)] = 0
    p = token_probs(torch.from_numpy(x)[None].cuda(), T, top_k).cpu().numpy()[0].astype(np.float64)
    w = np.exp(x.astype(np.float64) / T)
    far = (p > 0) & (x < 0)
    assert far.sum() >= (top_k or vocab) - 1
    off = p[far] / (w[far] / w.sum()) - 1
    step, rest, apart = 2.0 ** -18, 2.0 ** -22 + 2 * 2.0 ** -24 + 2.0 ** -40, far.sum()
    if not top_k:
        step, rest, apart = step + 2.0 ** -19, 2 * rest, apart / 1024
    assert np.abs(off).max() <= step * np.log(2) + rest
    assert abs(off.mean()) <= 6 * 2 * step * np.log(2) / np.sqrt(12 * apart) + rest
