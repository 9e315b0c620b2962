"""Scores and values of any size in range (mg_paged.h: "In range")."""
import numpy as np
import pytest

import paged_ref as ref
import paged_tight as tight
from gpu_util import say
from test_gpu_paged import kind_of
from test_gpu_paged_tight import attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("contract", ["fast_bf16", "strict_f32"])
@pytest.mark.parametrize("scale", [0.3, -1.7, 2.0 ** -30 / 3])
@pytest.mark.parametrize("B,Hq,H,Lq,d,page,key_len,listed", [
    (2, 4, 2, 3, 32, 16, [40, 9], False), (2, 8, 1, 5, 64, 64, [250, 700], False),
    (1, 8, 2, 1, 128, 16, [9000], False), (2, 8, 2, 2, 64, 32, [3000, 129], True)])
def test_scores_of_any_size(gpu_lib, B, Hq, H, Lq, d, page, key_len, listed, scale, contract):
    """Products are whole numbers times a power of two, so scores are exact; from 2^7 on
    one that is not the largest has no weight in f32."""
    say("paged range B%d Hq%d d%d %s scale %g %s" % (B, Hq, d, key_len, scale, contract))
    rng = np.random.default_rng(d + B)
    P, G, N = ref.pages(max(key_len), page), Hq // H, 30
    table = rng.integers(0, N, (B, P))
    K = rng.integers(-3, 4, (N, H, page, d)).astype(np.float32)
    K[..., 3:] = rng.integers(-200, 201, (N, H, page, d - 3))
    V = rng.integers(-1, 2, (N, H, page, d)).astype(np.float32)
    index = np.tile(np.arange(P), (B, H, Lq, 1)) if listed else None
    whole = rng.integers(1, 4, (B, Hq, Lq, 3)) * rng.choice([-1, 1], (B, Hq, Lq, 3))
    down = 2.0 ** np.ceil(np.log2(1 / abs(scale)))   # scores from 1 on, whatever the scale
    for power in (7, 20, 31, 40, 75, 90):
        Q = np.zeros((B, Hq, Lq, d), np.float32)
        Q[..., :3] = whole * 2.0 ** power * down
        O, LSE = attention(gpu_lib, Q, K, V, table, key_len, None, scale, contract, index)
        for b, hq, i in np.ndindex(B, Hq, Lq):
            j = np.arange(ref.limit(key_len[b], Lq, i, True))
            at = (table[b, j // page], hq // G, j % page)
            s = K[at].astype(np.float64) @ Q[b, hq, i].astype(np.float64) * np.float64(np.float32(scale))
            most = s == s.max()
            want = V[at][most].astype(np.float64).mean(0), s.max() + np.log(most.sum())
            off = tight.marked_off(O[b, hq, i][None], LSE[b, hq, i][None], want[0][None],
                                   np.array([want[1]]), kind_of(contract))
            assert not off.any(), (power, b, hq, i, O[b, hq, i][:4], LSE[b, hq, i], want[1])


@pytest.mark.parametrize("contract", ["fast_bf16", "strict_f32"])
@pytest.mark.parametrize("power", [-100, 103])
@pytest.mark.parametrize("B,Hq,H,Lq,d,page,P,key_len,listed", [
    (2, 8, 2, 3, 64, 16, 30, 477, False), (1, 16, 1, 1, 128, 64, 2000, 128000, False),
    (2, 8, 2, 1, 32, 128, 300, 38000, True)])
def test_values_of_any_size(gpu_lib, B, Hq, H, Lq, d, page, P, key_len, listed, power, contract):
    """Whole numbers times a power of two, added exactly (paged_tight.py)."""
    say("paged range of V 2^%d d%d %d tokens %s" % (power, d, key_len, contract))
    rng = np.random.default_rng(P)
    N, G, unit = 60, Hq // H, 2.0 ** power
    K, V = tight.marked_inputs(rng, N, H, page, d)
    V[:, :, 0] = 1   # sums grow with the length
    Q, channel = tight.marked_rows(rng, B, Hq, Lq, d)
    table = rng.integers(0, N, (B, P))
    index = np.tile(np.arange(P), (B, H, Lq, 1)) if listed else None
    O, LSE = attention(gpu_lib, Q, K, (V * unit).astype(np.float32), table, [key_len] * B, None, 1.0,
                       contract, index)
    for b, h, i in np.ndindex(B, H, Lq):
        j = np.arange(ref.limit(key_len, Lq, i, True))
        hq = slice(h * G, (h + 1) * G)
        want = tight.marked(K, V, table[b, j // page], j % page, h, channel[b, hq, i])
        off = tight.marked_off(O[b, hq, i] / unit, LSE[b, hq, i], *want, kind_of(contract))
        assert not off.any(), (b, h, i, O[b, hq, i] / unit - want[0])
