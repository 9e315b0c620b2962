"""Inputs of the paged attention whose results are known closely, and what they may be
off by.

Marked tokens.  A query row is 1 in one channel and 0 elsewhere; K is 0 or -1024
there, V is -1, 0 or 1.  With scale 1 a token's weight is then exactly 1 or 0
(exp(-1024) is 0 in f32, also as the factor of a unit whose tokens all have it), sums
are whole numbers (bf16: in steps of 2^-8, as 1 is 1 - 2^-8 and 2^-8) below 2^15, and
no order of them rounds.  LSE is the logarithm of a count, O a sum over that count:
one token too many or too few is seen at any length, and a page in another's place.

Weighted tokens.  Bounds from the roundings' own size, for errors that have nothing to
do with each other: they add as squares, not as magnitudes.
"""
import numpy as np

import paged_ref as ref

U = ref.HALF_STEP["f32"]
LOW = -1024.0
CHAIN = 2 ** 11   # roundings one after the other in a sum at most: terms of a lane, waves, units


def marked_inputs(rng, N, H, page, d):
    """K and V of the pools, of which both types hold every value; a page's first token
    counts in every channel, so that no row has none."""
    K = np.where(rng.random((N, H, page, d)) < 0.5, np.float32(LOW), np.float32(0))
    K[:, :, 0] = 0
    V = rng.integers(-1, 2, (N, H, page, d)) * (rng.random((N, H, page, d)) < 0.4)
    return K, V.astype(np.float32)


def marked_rows(rng, B, Hq, Lq, d):
    """Query rows and the channel that each of them looks at."""
    channel = rng.integers(0, d, (B, Hq, Lq))
    return np.eye(d, dtype=np.float32)[channel], channel


def marked(K, V, at, row, h, channel):
    """O and LSE of the rows that look at `channel` [r], over tokens at[i], row[i] of the
    pools: whole sums, divided once."""
    w = (K[at, h, row][:, channel] == 0).astype(np.float64)    # [tokens, r]
    n = w.sum(0)
    O = (w.T @ V[at, h, row].astype(np.float64)) / np.maximum(n, 1)[:, None]
    with np.errstate(divide="ignore"):
        return O, np.log(n)


def marked_off(O, LSE, want_O, want_LSE, kind):
    """Where O and LSE are not what exact sums give.  The count's reciprocal is within
    two half steps, the product rounds once, O is rounded to its type; the logarithm's
    two parts and their sum round three times at most."""
    bad = np.abs(O - want_O) > np.abs(want_O) * (ref.HALF_STEP[kind] + 4 * U)
    with np.errstate(invalid="ignore"):
        far = np.abs(LSE - want_LSE) > 4 * U * np.maximum(np.abs(want_LSE), 1)
    return bad.any(-1) | far | np.isnan(LSE) | (np.isneginf(LSE) != np.isneginf(want_LSE))


def weighted(q, k, v, scale, kind):
    """O and LSE of one row over k, v [n, d] in 64 bits, and what they may be off by:
    O's norm (f32) or each of its elements (bf16), and LSE.

    A token's score is a sum of d products, each rounded at the size of the sum so far,
    which is about S = sqrt(sum q^2 k^2).  With it, with the exponent's size and with the
    exponential's steps, its p is relatively off by e = (sqrt(d) S + 4 + |s| + max |s|) u.
    These errors are each token's own: in O they add to sqrt(sum (e p v)^2).  O's sum
    rounds at its own size, c = n + 16 times (no more than CHAIN): sqrt(c) u (|O| + 3
    sqrt(sum (p v)^2)).  bf16: p is in two parts, within 2^-15, and O is rounded.  Twice
    all that; six times for single elements."""
    q, k, v = (x.astype(np.float64) for x in (q, k, v))
    s = scale * (k @ q)
    top = s.max()
    p = np.exp(s - top)
    LSE = top + np.log(p.sum())
    p /= p.sum()
    S = abs(scale) * np.sqrt(((k * q) ** 2).sum(1))
    e = (np.sqrt(k.shape[1]) * S + 4 + np.abs(s) + np.abs(s).max()) * U
    part = 2.0 ** -15 if kind == "bf16" else 0.0
    O, spread = p @ v, np.sqrt(p ** 2 @ v ** 2)
    own = np.sqrt(((e + part) * p) ** 2 @ v ** 2)
    chain = np.sqrt(min(CHAIN, len(p) + 16)) * U
    sums = chain * (np.abs(O) + 3 * spread)
    tL = 2 * (np.sqrt(((e * p) ** 2).sum()) + chain) + 4 * U * abs(LSE)
    if kind == "bf16":
        return O, LSE, ref.HALF_STEP[kind] * np.abs(O) + 6 * (own + sums), tL
    return O, LSE, 2 * np.linalg.norm(own + sums) + U * np.linalg.norm(O), tL


def weighted_off(O, LSE, want, kind):
    rO, rL, tO, tL = want
    off = np.abs(O - rO)
    return abs(LSE - rL) > tL or np.isnan(LSE) or \
        not (np.all(off <= tO) if kind == "bf16" else np.linalg.norm(off) <= tO)
