"""The paged attention against results that are known closely (paged_tight.py): no
token lost, none twice, no page in another's place at any length, over units, table
windows and joins; and no more rounding than the contracts name."""
import math

import numpy as np
import pytest

import paged_ref as ref
import paged_tight as tight
from gpu_util import say
from test_gpu_paged import dev, dtype_of, host, ints, kind_of, rounded, rows, table_of

pytestmark = pytest.mark.gpu


def attention(mg, Q, Kp, Vp, table, key_len, q_len, scale, contract, index=None):
    import torch
    dt = dtype_of(contract)
    O = torch.full(Q.shape, math.nan, dtype=dt, device="cuda")
    LSE = torch.full(Q.shape[:3], math.nan, device="cuda")
    args = [dev(Q, dt), dev(Kp, dt), dev(Vp, dt), ints(table), ints(key_len)]
    kw = dict(causal=True, scale=scale, contract=contract)
    if index is None:
        mg.mg_attn_fwd_paged(*args, O, LSE, ints(q_len), **kw)
    else:
        mg.mg_attn_fwd_paged_sparse(*args, ints(index), O, LSE, ints(q_len), **kw)
    return host(O).astype(np.float64), host(LSE).astype(np.float64)


MARKED = [
    # B, Hq, H, Lq, d, page, P, key_len
    (1, 4, 4, 1, 64, 16, 16, [256]),
    (3, 8, 1, 1, 128, 64, 12, [0, 700, 33]),
    (1, 8, 2, 2, 128, 16, 400, [4999]),
    (70, 8, 4, 1, 64, 16, 40, [(37 * b) % 600 for b in range(70)]),
    (3, 4, 4, 2, 32, 64, 900, [50000, 57600, 1]),
    (2, 16, 1, 1, 128, 64, 2000, [90000, 128000]),
    (12, 16, 16, 1, 128, 16, 2600, [41595 - (b % 3) for b in range(12)]),   # long units
    (8, 8, 8, 1, 64, 16, 4096, [65536 - 4001 * b for b in range(8)]),
    (1, 24, 1, 2, 128, 256, 300, [76799]),             # 48 rows a cache head
    (1, 32, 2, 7, 64, 128, 300, [38000]),              # 112
    (1, 8, 1, 40, 32, 16, 1200, [19001]),              # 320
    (200, 4, 2, 1, 64, 16, 130, [(b * 7919) % 2080 for b in range(200)]),
    (700, 2, 1, 1, 32, 16, 700, [(b * 7919) % 90 if b != 333 else 11000 for b in range(700)]),
]


@pytest.mark.parametrize("contract", ["fast_bf16", "strict_f32"])
@pytest.mark.parametrize("B,Hq,H,Lq,d,page,P,key_len", MARKED)
def test_every_token_counts_once(gpu_lib, B, Hq, H, Lq, d, page, P, key_len, contract):
    say("paged marked B%d Hq%d H%d Lq%d d%d page%d P%d %s" % (B, Hq, H, Lq, d, page, P, contract))
    rng = np.random.default_rng(P + B)
    N, G = 60 if P > 60 else P, Hq // H
    K, V = tight.marked_inputs(rng, N, H, page, d)
    Q, channel = tight.marked_rows(rng, B, Hq, Lq, d)
    table = rng.integers(0, N, (B, P))
    O, LSE = attention(gpu_lib, Q, K, V, table, key_len, None, 1.0, contract)
    kind = kind_of(contract)
    for b in sorted({0, 1 % B, B // 2, B - 1, int(np.argmax(key_len))}):
        for h in range(H):
            for i in range(Lq):
                j = np.arange(ref.limit(key_len[b], Lq, i, True))
                hq = slice(h * G, (h + 1) * G)
                want = tight.marked(K, V, table[b, j // page], j % page, h, channel[b, hq, i])
                off = tight.marked_off(O[b, hq, i], LSE[b, hq, i], *want, kind)
                assert not off.any(), (b, h, i, LSE[b, hq, i] - want[1])


@pytest.mark.parametrize("contract", ["fast_bf16", "strict_f32"])
@pytest.mark.parametrize("B,Hq,H,Lq,d,page,P,key_len,keep", [
    (64, 16, 16, 1, 128, 16, 1400, 22400, 301), (2, 8, 2, 3, 64, 64, 900, 57001, 257),
    (1, 8, 2, 1, 32, 256, 200, 51111, 130), (3, 40, 1, 1, 64, 16, 90, 1433, 47)])
def test_every_listed_token_counts_once(gpu_lib, B, Hq, H, Lq, d, page, P, key_len, keep, contract):
    say("paged marked sparse B%d d%d page%d keep%d %s" % (B, d, page, keep, contract))
    rng = np.random.default_rng(P + B)
    N, G = 60, Hq // H
    K, V = tight.marked_inputs(rng, N, H, page, d)
    Q, channel = tight.marked_rows(rng, B, Hq, Lq, d)
    table = rng.integers(0, N, (B, P))
    index = np.sort(rng.permuted(np.tile(np.arange(P), (B, H, Lq, 1)), axis=3)[..., :keep], 3)
    O, LSE = attention(gpu_lib, Q, K, V, table, [key_len] * B, None, 1.0, contract, index)
    for b in sorted({0, B - 1}):
        for h, i in np.ndindex(H, Lq):
            j = (index[b, h, i][:, None] * page + np.arange(page)).flatten()
            j = j[j < ref.limit(key_len, Lq, i, True)]
            hq = slice(h * G, (h + 1) * G)
            want = tight.marked(K, V, table[b, j // page], j % page, h, channel[b, hq, i])
            off = tight.marked_off(O[b, hq, i], LSE[b, hq, i], *want, kind_of(contract))
            assert not off.any(), (b, h, i, LSE[b, hq, i] - want[1])


@pytest.mark.parametrize("contract", ["fast_bf16", "strict_f32"])
@pytest.mark.parametrize("B,Hq,H,Lq,d,page,key_len", [
    (2, 4, 2, 3, 32, 16, [40, 9]), (1, 8, 2, 1, 64, 32, [256]), (2, 8, 1, 5, 64, 64, [250, 700]),
    (2, 4, 4, 1, 128, 16, [700, 333]), (1, 40, 1, 2, 128, 64, [511]), (1, 4, 1, 1, 128, 64, [2000])])
def test_no_more_rounding_than_named(gpu_lib, B, Hq, H, Lq, d, page, key_len, contract):
    say("paged roundings B%d Hq%d d%d %s %s" % (B, Hq, d, key_len, contract))
    rng = np.random.default_rng(d + B)
    P, kind, scale = ref.pages(max(key_len), page), kind_of(contract), d ** -0.5
    N, table = table_of(rng, B, P, page, key_len)
    Kp, Vp = (rows(rng, (N, H, page, d), contract) for _ in range(2))
    Q = rounded(rng.standard_normal((B, Hq, Lq, d)), contract)
    O, LSE = attention(gpu_lib, Q, Kp, Vp, table, key_len, None, scale, contract)
    for b, hq, i in np.ndindex(B, Hq, Lq):
        j = np.arange(ref.limit(key_len[b], Lq, i, True))
        at = (table[b, j // page], hq // (Hq // H), j % page)
        want = tight.weighted(Q[b, hq, i], Kp[at], Vp[at], scale, kind)
        assert not tight.weighted_off(O[b, hq, i], LSE[b, hq, i], want, kind), \
            (b, hq, i, np.abs(O[b, hq, i] - want[0]).max(), LSE[b, hq, i] - want[1], want[2:])
