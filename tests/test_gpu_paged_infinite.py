"""V that is infinite or NaN in tokens which some rows see and others do not, for
every number of rows that a workgroup takes: each row has what its own tokens give."""
import numpy as np
import pytest

import paged_ref as ref
import paged_tight as tight
from gpu_util import say
from test_gpu_paged import kind_of, rounded, rows, table_of
from test_gpu_paged_tight import attention

pytestmark = pytest.mark.gpu


def of_specials(v):
    """What a column of weights above 0 makes of v's infinities and NaN [n, d]: 0 where
    there are none."""
    with np.errstate(invalid="ignore"):
        return np.where(np.isfinite(v), 0, v).sum(0)


CASES = [
    # G, Lq, d, page, P, key_len, q_len
    (3, 5, 64, 16, 30, [90, 21], [5, 4]),             # 15 rows a cache head
    (3, 10, 128, 16, 30, [100, 9], None),             # 30: two tiles a wave
    (12, 5, 32, 64, 9, [300, 33], None),              # 60: two waves share tokens
    (5, 24, 64, 32, 30, [777, 64], [24, 11]),         # 120: a wave for every 32 rows
    (4, 40, 128, 16, 40, [610, 40], [37, 40]),        # 160: two groups
    (7, 40, 32, 16, 60, [700, 41], None),             # 280, heads and tiles out of step
    (3, 10, 64, 64, 100, [5000, 3333], None),         # in the last of many units
    (5, 24, 128, 16, 400, [6001, 31], None),
    (4, 40, 64, 128, 40, [4999, 129], [40, 33]),
]


@pytest.mark.parametrize("contract", ["fast_bf16", "strict_f32"])
@pytest.mark.parametrize("G,Lq,d,page,P,key_len,q_len", CASES)
def test_special_values_behind_the_causal_mask(gpu_lib, G, Lq, d, page, P, key_len, q_len, contract):
    say("paged special V G%d Lq%d d%d page%d %s %s" % (G, Lq, d, page, key_len, contract))
    rng = np.random.default_rng(G * Lq + d)
    B, H, scale, kind = len(key_len), 2, d ** -0.5, kind_of(contract)
    q_len = [Lq] * B if q_len is None else q_len
    N, table = table_of(rng, B, P, page, key_len)
    Kp, Vp = (rows(rng, (N, H, page, d), contract) for _ in range(2))
    Q = rounded(rng.standard_normal((B, G * H, Lq, d)), contract)
    for b, n in enumerate(key_len):
        # in tokens of the last rows, and in one that all rows see
        first = max(n - q_len[b] + 1, 0)
        for j in sorted({n - 1, (first + n - 1) // 2, first, max(n - q_len[b] - 20, 0)}):
            for h in range(H):
                c = rng.permutation(d)[:4]
                Vp[table[b, j // page], h, j % page, c] = [np.inf, -np.inf, np.nan, np.inf]
    finite = np.where(np.isfinite(Vp), Vp, 0).astype(np.float32)
    O, LSE = attention(gpu_lib, Q, Kp, Vp, table, key_len, q_len, scale, contract)
    odd = 0
    for b, hq, i in np.ndindex(B, G * H, Lq):
        j = np.arange(ref.limit(key_len[b], q_len[b], i, True))
        if len(j) == 0:
            assert np.all(O[b, hq, i] == 0) and np.isneginf(LSE[b, hq, i])
            continue
        at = (table[b, j // page], hq // G, j % page)
        special = of_specials(Vp[at])
        assert np.array_equal(np.where(special == 0, 0, O[b, hq, i]), special, equal_nan=True), \
            (b, hq, i)
        want = tight.weighted(Q[b, hq, i], Kp[at], finite[at], scale, kind)
        got = np.where(special == 0, O[b, hq, i], want[0])
        assert not tight.weighted_off(got, LSE[b, hq, i], want, kind), (b, hq, i)
        odd += (special != 0).sum()
    assert odd > 0
