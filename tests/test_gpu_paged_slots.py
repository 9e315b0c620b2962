"""Rows of a page whose slots rise and leave some out (mg_paged.h: mg_paged_append):
the page's bounds cover every row that is written, wherever waves begin."""
import numpy as np
import pytest

import paged_ref as ref
from gpu_util import say
from test_gpu_paged import dev, dtype_of, host, ints, kind_of, rows

pytestmark = pytest.mark.gpu


def slots_with_gaps(rng, page, N, T, least, apart):
    """T slots: `least` rows or more of one page after another, each slot up to `apart`
    above the one before; some pages begin at row 0."""
    out = []
    for p in rng.permutation(N):
        at = 0 if rng.random() < 0.5 else int(rng.integers(0, page // 2))
        most = int(rng.integers(least, page + 1))
        while at < page and most > 0 and len(out) < T:
            out.append(int(p) * page + at)
            at += int(rng.integers(1, apart + 1))
            most -= 1
    assert len(out) == T
    return np.array(out)


@pytest.mark.parametrize("contract", ["fast_bf16", "strict_f32"])
@pytest.mark.parametrize("H,page,d,T", [
    (2, 16, 128, 2), (2, 16, 64, 70), (1, 64, 32, 300), (3, 256, 128, 700), (2, 128, 64, 90),
    (8, 16, 128, 2500), (8, 32, 64, 3000), (8, 64, 128, 2500), (2, 256, 32, 9000)])
def test_slots_that_rise_with_gaps(gpu_lib, H, page, d, T, contract):
    say("paged append with gaps H%d page%d d%d T%d %s" % (H, page, d, T, contract))
    rng = np.random.default_rng(T + page)
    N = T // (page // 8) + 3
    for apart in (2, 5):
        slot = slots_with_gaps(rng, page, N, T, page // 4, apart) if T > 2 else np.array([21, 23])
        K, V = rows(rng, (T, H, d), contract), rows(rng, (T, H, d), contract)
        Kp, Vp = (rows(rng, (N, H, page, d), contract) for _ in range(2))
        bounds = np.sort(rows(rng, (N, H, 2, d), contract), 2)
        g = [dev(x, dtype_of(contract)) for x in (K, V, Kp, Vp)]
        gb = dev(bounds, dtype_of(contract))
        gpu_lib.mg_paged_append(*g, ints(slot), gb, contract=contract)
        ref.append(K, V, Kp, Vp, bounds, slot, kind_of(contract))
        assert np.array_equal(host(g[2]), Kp) and np.array_equal(host(g[3]), Vp)
        assert np.array_equal(host(gb), bounds)
