"""Pages with a channel of NaN alone are chosen last (mg_paged.h: mg_paged_select)."""
import numpy as np
import pytest

import paged_ref as ref
from gpu_util import say
from test_gpu_paged import chosen, dev, dtype_of, host, ints, kind_of, on_grid, reference_pages

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("contract", ["fast_bf16", "strict_f32"])
@pytest.mark.parametrize("page,d", [(16, 32), (64, 128)])
def test_a_channel_of_nan_alone_takes_a_page_behind_the_others(gpu_lib, page, d, contract):
    say("paged select: channels of NaN page%d d%d %s" % (page, d, contract))
    rng = np.random.default_rng(page)
    P, dt = 30, dtype_of(contract)
    K = on_grid(rng, (P * page, 1, d))
    odd = [2, 11, 17]
    for k, p in enumerate(odd):
        K[p * page:(p + 1) * page, :, 3 + k] = np.nan
    K[5 * page:6 * page - 1, :, 4] = np.nan   # but for one token
    pool = lambda: np.zeros((P, 1, page, d), np.float32)
    Kp, Vp, bounds = pool(), pool(), np.zeros((P, 1, 2, d), np.float32)
    slot = np.arange(P * page)
    gb = dev(bounds, dt)
    gpu_lib.mg_paged_append(dev(K, dt), dev(K, dt), dev(Kp, dt), dev(Vp, dt), ints(slot), gb,
                            contract=contract)
    ref.append(K, K, Kp, Vp, bounds, slot, kind_of(contract))
    assert np.array_equal(host(gb), bounds)
    Q = on_grid(rng, (1, 2, 3, d))
    Q[:, :, :, 3:6] += np.where(Q[:, :, :, 3:6] >= 0, 1, -1)   # of either sign, never 0
    for keep in (5, P - len(odd), P - 1):
        args = (np.arange(P)[None], [P * page], None, False, page, keep, 0, 0)
        got = chosen(gpu_lib, Q, bounds, *args, contract)
        assert np.array_equal(got, reference_pages(Q, bounds, *args))
        assert np.isin(got, odd).sum((0, 1, 3)).tolist() == [max(0, keep - P + len(odd))] * 3
