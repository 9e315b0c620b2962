"""The score that mg_paged.h states is the one that the tests' plain implementation
computes, also for a page whose bounds are reversed (a channel of NaN alone)."""
import re

import numpy as np

import paged_ref as ref
import paper_2608_01563_amd as mg


def stated(q, lo, hi):
    """The header's formula for query rows q [G, d] and one page's lo, hi [d]."""
    with open(mg.PAGED_HEADER_PATH) as f:
        text = re.search(r"max over the group's heads g of\s+sum_c (.*)", f.read()).group(1)
    text = re.sub(r" (lo|hi)\[c\]", r" * \1", text.replace("Q[g][c]", "q"))
    return max(sum(eval(text, {"q": float(x), "lo": float(a), "hi": float(b), "max": max,
                               "min": min})
                   for x, a, b in zip(row, lo, hi)) for row in q)


def test_the_headers_score():
    rng = np.random.default_rng(1)
    d, most = 32, ref.MOST["bf16"]
    q = rng.integers(-9, 10, (3, d)).astype(np.float64)
    K = rng.integers(-9, 10, (16, 1, d)).astype(np.float32)
    for channel in (None, 0, 7):
        if channel is not None:
            K[:, :, channel] = np.nan
        Kp, bounds = np.zeros((1, 1, 16, d)), np.zeros((1, 1, 2, d))
        ref.append(K, K, Kp, Kp.copy(), bounds, np.arange(16), "bf16")
        lo, hi = bounds[0, 0]
        assert channel is None or (lo[channel], hi[channel]) == (most, -most)
        assert ref.scores(q, bounds[:, 0], np.array([0]), 1)[0] == np.float32(stated(q, lo, hi))
