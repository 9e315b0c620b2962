"""The 4-bit key/value cache on the GPU (mg_kv4.h) against the plain 64-bit
implementation in kv4_ref.py: bytes written, rows read back, attention of few
and many rows, accumulated weights, eviction, and a run of all together."""
import math

import numpy as np
import pytest

import kv4_ref as ref
from gpu_util import say

pytestmark = pytest.mark.gpu


def dev(x, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return t if dtype is None else t.to(dtype)


def dtype_of(contract):
    import torch
    return torch.bfloat16 if contract == "fast_bf16" else torch.float32


def host(t):
    import torch
    return t.float().cpu().numpy() if t.dtype == torch.bfloat16 else t.cpu().numpy()


def rows(rng, shape, contract):
    x = (rng.standard_normal(shape) * np.exp(rng.standard_normal(shape[-1])) +
         rng.standard_normal(shape[-1])).astype(np.float32)
    return ref.bf16_round(x) if contract == "fast_bf16" else x


def filled(rng, B, H, L, d):
    """A cache whose tokens all hold something, as the reference and as bytes."""
    c = ref.Cache(B, H, L, d)
    for b in range(B):
        for which in range(2):
            c.put(which, b, np.arange(L), rows(rng, (H, L, d), "strict_f32"))
    return c


APPEND = [
    # B, H, n, L, d, start, count
    (1, 1, 1, 1, 32, [0], [1]),
    (2, 3, 1, 40, 64, [0, 39], None),
    (3, 2, 5, 50, 128, [0, 6, 45], [5, 3, 5]),
    (2, 2, 33, 64, 32, [31, 0], [33, 0]),
    (2, 1, 17, 30, 64, [-4, 20], [17, 17]),          # rows before 0 and behind L are dropped
    (2, 2, 100, 100, 128, None, [1, 100]),
    (1, 2, 70, 200, 128, [2147483647], None),        # far outside: nothing is written
    (1, 2, 70, 200, 64, [-2147483648], [2147483647]),
    (4, 1, 8, 64, 32, [0, 8, 9, 56], [-3, 8, 99, 8]),
]


@pytest.mark.parametrize("contract", ["fast_bf16", "strict_f32", "accelerated"])
@pytest.mark.parametrize("B,H,n,L,d,start,count", APPEND)
def test_append_and_read(gpu_lib, B, H, n, L, d, start, count, contract):
    import torch
    mg = gpu_lib
    say("kv4 append B%d H%d n%d L%d d%d %s" % (B, H, n, L, d, contract))
    rng = np.random.default_rng(n * 1000 + d)
    K, V = (rows(rng, (B, H, n, d), contract) for _ in range(2))
    want = filled(rng, B, H, L, d)
    raw = dev(want.to_bytes())
    weight = rng.random((B, H, L)).astype(np.float32)
    dw = dev(weight)
    ints = lambda x: None if x is None else dev(np.array(x, np.int32))
    st, ct = start or [0] * B, count or [n] * B
    dt = dtype_of(contract)
    mg.mg_kv4_append(dev(K, dt), dev(V, dt), raw, ints(start), ints(count), L=L, weight=dw,
                     contract=contract)
    ref.append(want, weight, K, V, st, ct)
    assert np.array_equal(host(raw), want.to_bytes())      # every byte, untouched tokens too
    assert np.array_equal(host(dw), weight)

    outK, outV = (torch.full((B, H, n, d), 7.0, dtype=dt, device="cuda") for _ in range(2))
    mg.mg_kv4_read(raw, outK, outV, ints(start), ints(count), L=L, contract=contract)
    for which, out in ((0, outK), (1, outV)):
        x = np.full((B, H, n, d), 7.0)
        vals = want.rows(which)
        for b in range(B):
            for j in range(min(max(ct[b], 0), n)):
                if 0 <= st[b] + j < L:
                    x[b, :, j] = vals[b, :, st[b] + j]
        x = x.astype(np.float32)   # one fma in f32, exact: 12 bits times 1 plus 8 bits
        tol = 2.0 ** -24 if contract != "fast_bf16" else 2.0 ** -8
        assert np.all(np.abs(host(out) - x) <= tol * np.abs(x))


def test_append_special_groups(gpu_lib):
    """Equal values, ties, zeros, subnormals, ranges beyond f32, infinities and NaN."""
    mg = gpu_lib
    say("kv4 append special groups")
    d, L = 128, 16
    K = np.zeros((1, 1, L, d), np.float32)
    K[0, 0, 0] = 3.25                                     # scale 0
    K[0, 0, 1] = (np.arange(d) % 31) * 0.5                # every second one a tie
    K[0, 0, 2] = -(np.arange(d) % 31) * 0.5
    K[0, 0, 3, :64] = 1e-40 * (np.arange(64) % 16)        # subnormal
    K[0, 0, 4, 5] = np.inf
    K[0, 0, 5, 70] = np.nan
    K[0, 0, 6, :2] = (3e38, -3e38)                        # range above f32
    K[0, 0, 7, 64] = -np.inf
    K[0, 0, 8] = np.float32(3.4e38)                       # minimum beyond bf16
    K[0, 0, 9] = np.linspace(-1, 1, d)
    K[0, 0, 10] = 2.0 ** -100 * np.linspace(0, 1, d)
    K[0, 0, 11, 3] = 2.0 ** 120
    K[0, 0, 12] = np.where(np.arange(d) % 2, 2.0 ** 60, 2.0 ** -60)
    K[0, 0, 13] = -0.0
    want = ref.Cache(1, 1, L, d)
    raw = dev(want.to_bytes())
    mg.mg_kv4_append(dev(K), dev(-K), raw, L=L, contract="strict_f32")
    ref.append(want, None, K, -K, [0], [L])
    got = ref.Cache.from_bytes(host(raw), 1, 1, L, d)
    for which in range(2):
        assert np.array_equal(got.code[which], want.code[which]), which
        a, b = got.rows(which), want.rows(which)
        assert np.array_equal(np.isnan(a), np.isnan(b))
        assert np.array_equal(a[~np.isnan(a)], b[~np.isnan(b)])
    assert np.isnan(want.rows(0)[0, 0, 4, :64]).all() and not np.isnan(want.rows(0)[0, 0, 4, 64:]).any()


ATTN = [
    # B, Hq, H, Lq, L, d, key_len, q_len, causal
    (1, 1, 1, 1, 1, 32, None, None, True),
    (1, 4, 4, 1, 256, 64, None, None, True),
    (2, 6, 2, 1, 31, 128, [31, 1], None, False),
    (3, 8, 1, 1, 700, 128, [0, 700, 33], None, True),
    (2, 4, 2, 3, 100, 64, [100, 2], [3, 3], True),      # a first row that sees nothing
    (2, 6, 3, 7, 201, 32, [201, 64], [7, 2], True),
    (2, 2, 2, 5, 64, 128, [40, 64], [5, 0], False),
    (1, 3, 1, 50, 333, 64, [300], None, True),
    (2, 4, 1, 37, 160, 128, [160, 37], [30, 37], True),
    (1, 2, 1, 150, 130, 32, None, None, True),          # more rows than tokens
    (1, 2, 2, 129, 500, 128, [470], None, False),
    (2, 8, 8, 1, 2000, 64, [2000, 77], None, True),     # split over workgroups
    (1, 8, 2, 2, 5000, 128, [4999], None, True),
    (1, 16, 1, 17, 600, 64, None, [11], True),
    (2, 4, 1, 16, 97, 64, [97, 0], None, True),         # many rows: short, and none at all
    (1, 8, 1, 70, 31, 128, None, [64], False),
    (2, 3, 1, 100, 1000, 32, [1000, 65], [100, 1], True),
    (1, 4, 2, 300, 640, 128, [639], [299], True),
    (1, 1, 1, 64, 6000, 64, [5990], None, True),        # split over workgroups
    (32, 8, 8, 257, 257, 32, None, None, True),
    (32, 8, 8, 300, 64, 128, None, None, False),
]


def many_rows(heads, rows, L):
    """Whether a bf16 call runs in the form for many rows and much work."""
    return rows >= 128 and heads * rows * L >= 1 << 25


MANY = [
    (2, 8, 2, 301, 7001, 128, [7001, 65], [301, 100], True),
    (1, 16, 16, 2100, 1001, 32, None, None, False),
    (32, 8, 8, 257, 511, 64, [511, 1, 0, 64, 65, 300, 2, 511] * 4,
     [257, 257, 3, 1, 200, 0, 257, 256] * 4, True),
    (1, 8, 1, 129, 32600, 64, [32577], None, True),
    (1, 2, 1, 65, 1 << 18, 32, [250001], None, False),
    (3, 3, 3, 4000, 2800, 128, [2800, 0, 5], [4000, 17, 0], True),
    (1, 1, 1, 128, 1 << 18, 128, [63], [127], True),
]


def reference(c, Q, kl, ql, G, causal, scale, strict):
    B, Hq, Lq, d = Q.shape
    H, L = c.dims[1], c.dims[2]
    O, tO = np.zeros(Q.shape), np.zeros(Q.shape)
    LSE, tL = np.zeros(Q.shape[:3]), np.zeros(Q.shape[:3])
    W, tW = np.zeros((B, H, L)), np.zeros((B, H, L))
    grp = [c.group(i) for i in range(2)]
    for b in range(B):
        n, r = min(max(kl[b], 0), L), min(max(ql[b], 0), Lq)
        for hq in range(Hq):
            h = hq // G
            out = ref.attention(Q[b, hq].astype(np.float64), [x[b, h] for x in c.code],
                                [(s[b, h], m[b, h]) for s, m in grp], n, r, causal, scale, strict,
                                not strict and many_rows(B * H, G * Lq, L))
            O[b, hq], LSE[b, hq], P, tO[b, hq], tL[b, hq], tP = out
            W[b, h, :n] += P.sum(0)
            tW[b, h, :n] += tP.sum(0)
    return O, LSE, W, tO, tL, tW


def check_attention(mg, rng, c, raw, Q, key_len, q_len, causal, scale, contract, weights):
    import torch
    B, Hq, Lq, d = Q.shape
    _, H, L, _ = c.dims
    dt = dtype_of(contract)
    kl, ql = key_len or [L] * B, q_len or [Lq] * B
    ints = lambda x: None if x is None else dev(np.array(x, np.int32))
    w0 = rng.random((B, H, L)).astype(np.float32)
    weight = dev(w0) if weights else None
    O = torch.full(Q.shape, math.nan, dtype=dt, device="cuda")
    LSE = torch.full(Q.shape[:3], math.nan, device="cuda")
    mg.mg_attn_fwd_kv4(dev(Q, dt), raw, O, LSE, ints(key_len), ints(q_len), H=H, L=L,
                       causal=causal, scale=scale, weight=weight, contract=contract)
    rO, rL, rW, tO, tL, tW = reference(c, Q, kl, ql, Hq // H, causal, scale,
                                       contract != "fast_bf16")
    gO, gL = host(O).astype(np.float64), host(LSE).astype(np.float64)
    assert np.array_equal(np.isneginf(rL), np.isneginf(gL))
    assert np.all(gO[np.isneginf(rL)] == 0)
    fin = ~np.isneginf(rL)
    assert np.all(np.abs(gL - rL)[fin] <= tL[fin]), (np.abs(gL - rL)[fin] / tL[fin]).max()
    assert np.all(np.abs(gO - rO) <= tO), (np.abs(gO - rO) / np.maximum(tO, 1e-300)).max()
    if weights:
        gW = host(weight).astype(np.float64)
        assert np.all(np.abs(gW - (w0 + rW)) <= tW + 2.0 ** -22 * (w0 + rW))
        for b in range(B):   # tokens behind the sequence keep their weights
            n = min(max(kl[b], 0), L)
            assert np.array_equal(gW[b, :, n:], w0[b, :, n:].astype(np.float64))


@pytest.mark.parametrize("contract,weights", [("fast_bf16", False), ("fast_bf16", True),
                                              ("strict_f32", True)])
@pytest.mark.parametrize("B,Hq,H,Lq,L,d,key_len,q_len,causal", ATTN)
def test_attention(gpu_lib, B, Hq, H, Lq, L, d, key_len, q_len, causal, contract, weights):
    say("kv4 attention B%d Hq%d H%d Lq%d L%d d%d %s weights=%s"
        % (B, Hq, H, Lq, L, d, contract, weights))
    rng = np.random.default_rng(Lq * 7919 + L * 31 + d)
    c = filled(rng, B, H, L, d)
    # what lies behind the sequences must not matter: NaN scales, any codes
    kl = key_len or [L] * B
    for b in range(B):
        for which in range(2):
            c.word[which][b][:, kl[b]:] = 0x7fc07fc0
            c.code[which][b][:, kl[b]:] = rng.integers(0, 16, c.code[which][b][:, kl[b]:].shape)
    Q = rows(rng, (B, Hq, Lq, d), contract)
    check_attention(gpu_lib, rng, c, dev(c.to_bytes()), Q, key_len, q_len, causal,
                    (-0.5 if L == 333 else 1.0) / math.sqrt(d), contract, weights)


@pytest.mark.parametrize("d", [32, 128])
def test_strict_parts_belong_together(gpu_lib, d):
    """Few tokens of nearly equal probability leave bounds of some 1e-5; of 10^5
    probabilities some lie next to a tie of f16, where the first part must be the
    one that the second was taken from (else O is off by up to 1e-4)."""
    say("kv4 strict, parts of probabilities d%d" % d)
    rng = np.random.default_rng(12)
    c = filled(rng, 1, 1, 8, d)
    Q = rows(rng, (1, 8, 2000, d), "strict_f32")
    check_attention(gpu_lib, rng, c, dev(c.to_bytes()), Q, None, None, False, 1e-2, "strict_f32",
                    False)


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("B,Hq,H,Lq,L,d,key_len,q_len,causal", MANY)
def test_attention_of_many_rows(gpu_lib, B, Hq, H, Lq, L, d, key_len, q_len, causal, weights):
    assert many_rows(B * H, Hq // H * Lq, L)
    test_attention(gpu_lib, B, Hq, H, Lq, L, d, key_len, q_len, causal, "fast_bf16", weights)


@pytest.mark.parametrize("contract,Lq,L", [("fast_bf16", 9, 900), ("strict_f32", 9, 900),
                                           ("fast_bf16", 130, 65000)])
def test_attention_over_a_wide_range(gpu_lib, contract, Lq, L):
    """Token scales and query rows of very different size, growing and falling
    along the sequence (the running units move both ways)."""
    say("kv4 attention, wide range %s Lq%d" % (contract, Lq))
    rng = np.random.default_rng(5)
    B, H, d = 1, 2, 64
    c = ref.Cache(B, H, L, d)
    size = np.exp(3.0 * np.sin(np.arange(L) / 40.0))[None, :, None]
    size[:, 500:520] = 1e4
    c.put(0, 0, np.arange(L), rows(rng, (H, L, d), "strict_f32"))
    c.put(1, 0, np.arange(L), (rows(rng, (H, L, d), "strict_f32") * size).astype(np.float32))
    Q = rows(rng, (B, 4, Lq, d), contract)
    Q[0, :, 3] *= 2.0 ** -40
    Q[0, :, 4] *= 2.0 ** 4
    Q[0, :, 5] = 0
    check_attention(gpu_lib, rng, c, dev(c.to_bytes()), Q, None, None, True, 0.3, contract, True)


@pytest.mark.parametrize("contract,Lq,L", [("fast_bf16", 3, 70), ("strict_f32", 3, 70),
                                           ("fast_bf16", 256, 65600)])
@pytest.mark.parametrize("size", [0.0, 1e-30, 1.0, 1e6, 2.0 ** 100])
def test_attention_of_flat_values(gpu_lib, contract, Lq, L, size):
    """V rows whose channels are all the same have scale 0: only minima."""
    say("kv4 attention, flat values of %g, %s Lq%d" % (size, contract, Lq))
    rng = np.random.default_rng(14)
    H, d = 1, 32
    c = ref.Cache(1, H, L, d)
    c.put(0, 0, np.arange(L), rows(rng, (H, L, d), "strict_f32"))
    flat = ref.bf16_round((size * rng.standard_normal((H, L, 1))).astype(np.float32))
    flat[:, :L // 3] = 0
    c.put(1, 0, np.arange(L), np.broadcast_to(flat, (H, L, d)).astype(np.float32))
    assert not c.group(1)[0].any()
    Q = rows(rng, (1, 2, Lq, d), contract)
    check_attention(gpu_lib, rng, c, dev(c.to_bytes()), Q, None, None, True, 0.2, contract, False)


@pytest.mark.parametrize("contract,Lq,L", [("fast_bf16", 3, 70), ("strict_f32", 3, 70),
                                           ("fast_bf16", 40, 70), ("strict_f32", 40, 70),
                                           ("fast_bf16", 256, 65600)])
@pytest.mark.parametrize("q,k,scale", [(1.0, 1.0, 0.0), (1e25, 1.0, -3e-26), (1e-30, 1.0, 3e29),
                                       (1.0, 1e20, 3e-21), (1.0, 1e-20, 3e19), (0.0, 1.0, 0.3)])
def test_attention_of_large_and_small_factors(gpu_lib, contract, Lq, L, q, k, scale):
    say("kv4 attention q %g k %g scale %g %s Lq%d" % (q, k, scale, contract, Lq))
    rng = np.random.default_rng(15)
    H, d = 1, 64
    c = filled(rng, 1, H, L, d)
    c.put(0, 0, np.arange(L), (k * rng.standard_normal((H, L, d))).astype(np.float32))
    Q = ref.bf16_round((q * rng.standard_normal((1, 2, Lq, d))).astype(np.float32))
    check_attention(gpu_lib, rng, c, dev(c.to_bytes()), Q, None, None, True, scale, contract, True)


@pytest.mark.parametrize("contract,value", [("fast_bf16", 0.0), ("strict_f32", 3.0)])
def test_the_longest_sequence(gpu_lib, contract, value):
    """2^24 tokens of equal score: O is their value, LSE the logarithm of their
    number, and each gathers 2^-24."""
    import torch
    mg = gpu_lib
    say("kv4 attention over 2^24 tokens %s" % contract)
    L, d, n = 1 << 24, 32, 1 << 22
    dt = dtype_of(contract)
    cache, w = mg.kv4_cache(1, 1, L, d), torch.zeros(1, 1, L, device="cuda")
    V = torch.full((1, 1, n, d), value, dtype=dt, device="cuda")
    for at in range(0, L, n):
        mg.mg_kv4_append(V, V, cache, dev(np.array([at], np.int32)), L=L, contract=contract)
    Q = torch.zeros(1, 2, 1, d, dtype=dt, device="cuda")
    O, LSE = mg.attention_forward_kv4(Q, cache, H=1, L=L, causal=True, scale=1.0, weight=w,
                                      contract=contract)
    # equal addends, in partial sums of fewer than 2^18 of them: 2^-7 at the very worst
    assert np.all(np.abs(host(O) - value) <= 2.0 ** -7 * value)
    assert np.all(np.abs(host(LSE) - 24 * math.log(2)) <= 2.0 ** -7)
    assert np.all(np.abs(host(w) * 2.0 ** 23 - 1) <= 2.0 ** -7)


@pytest.mark.parametrize("contract", ["fast_bf16", "strict_f32"])
@pytest.mark.parametrize("Lq,L", [(1, 100), (20, 100), (40, 100), (512, 32768)])
def test_attention_not_a_number(gpu_lib, contract, Lq, L):
    """A NaN token reaches the rows that see it, and its own group's channels of
    O if only its V is NaN; rows that do not see it are as without it."""
    import torch
    mg = gpu_lib
    say("kv4 attention with NaN %s Lq%d" % (contract, Lq))
    rng = np.random.default_rng(6)
    B, H, d = 1, 1, 128
    n = L - 10
    c = filled(rng, B, H, L, d)
    dt = dtype_of(contract)
    Q = dev(rows(rng, (B, 2, Lq, d), contract), dt)

    def run(cache):
        return [host(t) for t in mg.attention_forward_kv4(
            Q, dev(cache.to_bytes()), H=H, L=L, causal=True, scale=0.1,
            key_len=dev(np.array([n], np.int32)), contract=contract)]

    O, LSE = run(c)
    at = n - (1 if Lq == 1 else 10)   # rows from at on see token `at`
    first = 0 if Lq == 1 else Lq - 10
    c.word[1][0, 0, at, 1] = 0x7fc07fc0
    O2, LSE2 = run(c)
    assert np.array_equal(O2[:, :, :first], O[:, :, :first]) and np.array_equal(LSE2, LSE)
    assert np.isnan(O2[:, :, first:, 64:]).all()
    assert np.array_equal(O2[:, :, first:, :64], O[:, :, first:, :64])
    c.word[0][0, 0, at, 0] = 0x7fc07fc0
    O3, LSE3 = run(c)
    assert np.array_equal(O3[:, :, :first], O[:, :, :first])
    assert np.isnan(O3[:, :, first:]).all() and np.isnan(LSE3[:, :, first:]).all()


EVICT = [
    # B, H, L, d, keep, recent, key_len
    (1, 1, 1, 32, 1, 0, None),
    (2, 2, 50, 64, 20, 5, [50, 20]),
    (2, 1, 100, 128, 99, 99, [100, 0]),
    (1, 3, 333, 32, 1, 1, None),
    (1, 2, 333, 128, 7, 0, [300]),
    (2, 2, 3000, 64, 1500, 100, [2999, 1501]),
    (1, 2, 5000, 128, 2300, 31, None),
    (1, 1, 20001, 32, 9000, 3000, [19999]),
    (1, 1, 40000, 32, 20011, 7, None),       # more than a workgroup keeps in registers
]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,H,L,d,keep,recent,key_len", EVICT)
def test_evict(gpu_lib, B, H, L, d, keep, recent, key_len, in_place):
    import torch
    mg = gpu_lib
    say("kv4 evict B%d H%d L%d d%d keep%d in_place=%s" % (B, H, L, d, keep, in_place))
    rng = np.random.default_rng(L + keep)
    Lp = (L + 31) // 32 * 32
    c, o = ref.Cache(B, H, L, d), ref.Cache(B, H, L, d)
    for x in (c, o):
        for which in range(2):
            x.code[which] = rng.integers(0, 16, (B, H, Lp, d)).astype(np.uint8)
            x.word[which] = rng.integers(0, 2 ** 32, x.word[which].shape).astype(np.uint32)
    # many equal weights, zeros of both signs, some NaN, an infinity
    w = rng.integers(0, 40, (B, H, L)).astype(np.float32) / 8
    w[rng.random(w.shape) < 0.1] = -0.0
    w[rng.random(w.shape) < 0.03] = np.nan
    w[..., L // 2] = np.inf
    w[..., L // 3] = -1.5
    ow = rng.random((B, H, L)).astype(np.float32)
    want, want_w = (c, w.copy()) if in_place else (o, ow.copy())
    raw, dw = dev(c.to_bytes()), dev(w)
    out = None if in_place else dev(o.to_bytes())
    dow = None if in_place else dev(ow)
    index = torch.full((B, H, keep), -7, dtype=torch.int32, device="cuda")
    kl = None if key_len is None else dev(np.array(key_len, np.int32))
    new = torch.full((B,), -7, dtype=torch.int32, device="cuda") if not in_place or kl is None \
        else kl   # the lengths may be cut in place too
    mg.mg_kv4_evict(raw, dw, index, new, kl, d=d, recent=recent, out_cache=out, out_weight=dow)
    src = ref.Cache.from_bytes(c.to_bytes(), B, H, L, d)
    want_i = np.full((B, H, keep), -1)
    for b in range(B):
        n = L if key_len is None else key_len[b]
        for h in range(H):
            at = ref.evict(w[b, h], n, keep, recent)
            m = len(at)
            want_i[b, h, :m] = at
            for which in range(2):
                want.code[which][b, h, :m] = src.code[which][b, h, at]
                want.word[which][b, h, :m] = src.word[which][b, h, at]
            want_w[b, h, :m] = w[b, h, at]
    assert np.array_equal(host(new), [min(keep, L if key_len is None else k)
                                      for k in (key_len or [L] * B)])
    assert np.array_equal(host(index), want_i)
    got_w = host(dw if in_place else dow)
    assert np.array_equal(got_w, want_w, equal_nan=True)
    assert np.array_equal(host(raw if in_place else out), want.to_bytes())
    if not in_place:
        assert np.array_equal(host(raw), c.to_bytes())


@pytest.mark.parametrize("L,keep,recent", [(9000, 4000, 10), (30000, 12000, 0), (33000, 100, 50)])
def test_evict_by_weights_of_every_kind(gpu_lib, L, keep, recent):
    """All weights equal, all NaN, spread over the whole range, negative, and
    few above many."""
    import torch
    mg = gpu_lib
    say("kv4 evict L%d, weights of every kind" % L)
    rng = np.random.default_rng(L)
    bits = rng.integers(0, 1 << 32, L, dtype=np.uint32).view(np.float32)   # NaN and inf too
    w = np.stack([np.full(L, 0.125), np.full(L, np.nan), bits,
                  -np.exp(rng.standard_normal(L)),
                  np.where(rng.random(L) < 0.01, 2.0, 1e-30 * rng.random(L))]).astype(np.float32)
    H = len(w)
    cache = mg.kv4_cache(1, H, L, 32)
    index = torch.empty(1, H, keep, dtype=torch.int32, device="cuda")
    mg.mg_kv4_evict(cache, dev(w[None]), index, dev(np.zeros(1, np.int32)), d=32, recent=recent)
    for h in range(H):
        assert np.array_equal(host(index)[0, h], ref.evict(w[h], L, keep, recent)), h


@pytest.mark.parametrize("contract", ["fast_bf16", "strict_f32"])
def test_a_served_sequence(gpu_lib, contract):
    """Prompt, decode steps, eviction, more steps: after each, attention and
    weights against the reference's own cache."""
    import torch
    mg = gpu_lib
    say("kv4 served sequence %s" % contract)
    rng = np.random.default_rng(11)
    B, Hq, H, L, d = 2, 4, 2, 96, 64
    keep, recent = 24, 6
    dt = dtype_of(contract)
    cache = mg.kv4_cache(B, H, L, d)
    cache.fill_(0xff)                       # nothing may depend on what was there
    weight = torch.full((B, H, L), math.nan, device="cuda")
    length = torch.zeros(B, dtype=torch.int32, device="cuda")
    index = torch.empty(B, H, keep, dtype=torch.int32, device="cuda")
    c = ref.Cache.from_bytes(host(cache), B, H, L, d)
    n = np.zeros(B, int)
    w, tol = np.zeros((B, H, L)), np.zeros((B, H, L))

    def step(m, count):
        K, V = (rows(rng, (B, H, m, d), contract) for _ in range(2))
        Q = rows(rng, (B, Hq, m, d), contract)
        mg.mg_kv4_append(dev(K, dt), dev(V, dt), cache, length, dev(np.array(count, np.int32)),
                         L=L, weight=weight, contract=contract)
        ref.append(c, None, K, V, n, count)
        length.add_(dev(np.array(count, np.int32)))
        n[:] += count
        O, LSE = mg.attention_forward_kv4(dev(Q, dt), cache, H=H, L=L, causal=True, scale=0.125,
                                          key_len=length, q_len=dev(np.array(count, np.int32)),
                                          weight=weight, contract=contract)
        rO, rL, rW, tO, tL, tW = reference(c, Q, n, count, Hq // H, True, 0.125,
                                           contract != "fast_bf16")
        fin = ~np.isneginf(rL)
        assert np.all(np.abs(host(O) - rO) <= tO)
        assert np.all(np.abs(host(LSE) - rL)[fin] <= tL[fin])
        w.__iadd__(rW)
        tol.__iadd__(tW + 2.0 ** -23 * w)
        for b in range(B):
            assert np.all(np.abs(host(weight)[b, :, :n[b]] - w[b, :, :n[b]]) <= tol[b, :, :n[b]])

    step(40, [40, 23])
    for _ in range(3):
        step(1, [1, 1])
    mg.mg_kv4_evict(cache, weight, index, length, length, d=d, recent=recent)
    kept = host(index)
    for b in range(B):
        m = min(n[b], keep)
        for h in range(H):
            at = kept[b, h, :m]
            # weights that differ by more than their bounds are in the right order
            old = np.arange(n[b] - recent)
            gone = np.setdiff1d(old, at)
            stay = np.intersect1d(old, at)
            if len(gone) and len(stay):
                assert (w + tol)[b, h, stay].min() >= (w - tol)[b, h, gone].max()
            assert np.array_equal(at[m - recent:], np.arange(n[b] - recent, n[b]))
            for which in range(2):
                c.code[which][b, h, :m] = c.code[which][b, h, at]
                c.word[which][b, h, :m] = c.word[which][b, h, at]
            w[b, h, :m], tol[b, h, :m] = w[b, h, at], tol[b, h, at]
        w[b, :, m:], tol[b, :, m:] = 0, 0
        n[b] = m
    assert np.array_equal(host(length), n)
    for _ in range(2):
        step(1, [1, 1])
    step(5, [5, 2])
