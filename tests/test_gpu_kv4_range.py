"""Attention over the 4-bit cache at the ends of its range: values far above
the others behind what a row sees."""
import numpy as np
import pytest

import kv4_ref as ref
from gpu_util import say
from test_gpu_kv4 import check_attention, dev, dtype_of, filled, host, many_rows, rows

pytestmark = pytest.mark.gpu

# kv4_many holds values in units of up to 2^12 of what a row itself sees, beside
# the 2^-34 of them that the reference's bound has for those units
MANY_UNITS = 2.0 ** (12 - 34)


def check_rows_before(c, Q, O, LSE, n, cuts, causal_scale, strict, heads=None):
    """Rows between the tokens `cuts`, which are out of the ordinary, against the
    reference over the tokens that they can see: a token that a row does not see
    must not widen its bound."""
    B, Hq, Lq, d = Q.shape
    H = c.dims[1]
    many = not strict and many_rows(B * H, Hq // H * Lq, c.dims[2])
    O, LSE = host(O).astype(np.float64), host(LSE).astype(np.float64)
    done = 0
    for cut in list(cuts) + [n]:
        m = cut - (n - Lq)      # rows that do not see token `cut`
        for hq in heads or range(Hq):
            h = hq // (Hq // H)
            rO, rL, _, tO, tL, _ = ref.attention(
                Q[0, hq, :m].astype(np.float64), [x[0, h] for x in c.code],
                [tuple(p[0, h] for p in c.group(i)) for i in range(2)], cut, m, True,
                causal_scale, strict, many)
            if many:
                tO = tO + MANY_UNITS * np.abs(c.rows(1)[0, h, :cut]).max()
            off = np.abs(O[0, hq, done:m] - rO[done:])
            assert np.all(off <= tO[done:]), (cut, hq, (off / tO[done:]).max())
            assert np.all(np.abs(LSE[0, hq, done:m] - rL[done:]) <= tL[done:]), (cut, hq)
        done = m


def run(mg, c, Q, n, scale, contract):
    return mg.attention_forward_kv4(dev(Q, dtype_of(contract)), dev(c.to_bytes()), H=c.dims[1],
                                    L=c.dims[2], causal=True, scale=scale,
                                    key_len=dev(np.array([n], np.int32)), contract=contract)


@pytest.mark.parametrize("contract", ["fast_bf16", "strict_f32"])
@pytest.mark.parametrize("grow", [20, 60])
@pytest.mark.parametrize("Hq,H,Lq,L,d,cuts", [
    (2, 1, 5, 70, 64, [68]),                  # the last of few rows sees it alone
    (4, 2, 7, 400, 128, [394, 398]),          # two, one above the other
    (3, 1, 50, 333, 32, [300, 301, 331]),
    (1, 1, 40, 40, 64, [1, 17, 39]),          # the first row sees one token
    (2, 2, 3, 5000, 128, [4998])])            # split over workgroups
def test_values_that_rows_do_not_see(gpu_lib, contract, grow, Hq, H, Lq, L, d, cuts):
    """Tokens whose V is 2^20 or 2^60 times the others (and the next one that
    again) must not cost the rows before them anything."""
    say("kv4 attention, unseen values 2^%d, %s Hq%d Lq%d L%d d%d" % (grow, contract, Hq, Lq, L, d))
    rng = np.random.default_rng(grow + L + d)
    c = filled(rng, 1, H, L, d)
    for k, cut in enumerate(cuts):
        big = rows(rng, (H, 1, d), "strict_f32") * 2.0 ** (grow * (k + 1) / len(cuts))
        c.put(1, 0, np.array([cut]), big.astype(np.float32))
    n = L - 1 if L - 1 not in cuts else L
    Q = rows(rng, (1, Hq, Lq, d), contract)
    O, LSE = run(gpu_lib, c, Q, n, 0.1, contract)
    check_rows_before(c, Q, O, LSE, n, cuts, 0.1, contract != "fast_bf16")


@pytest.mark.parametrize("contract", ["fast_bf16", "strict_f32"])
@pytest.mark.parametrize("first,at", [(-70, 650), (-70, 400), (-30, 130), (0, 699)])
def test_a_leap_of_values(gpu_lib, contract, first, at):
    """One V 2^150 (or as far as values may go) above those before it must leave LSE,
    which V has no part in, and the probabilities as they are."""
    say("kv4 attention, a leap of values at %d from 2^%d, %s" % (at, first, contract))
    rng = np.random.default_rng(at)
    H, L, d = 2, 700, 64
    c = filled(rng, 1, H, L, d)
    x = (rows(rng, (H, L, d), "strict_f32") * 2.0 ** first).astype(np.float32)
    x[:, at] = rows(rng, (H, d), "strict_f32") * np.float32(2.0 ** min(80, first + 150))
    c.put(1, 0, np.arange(L), x)
    Q = rows(rng, (1, 4, 2, d), contract)
    check_attention(gpu_lib, rng, c, dev(c.to_bytes()), Q, None, None, False, 0.1, contract, True)


@pytest.mark.parametrize("grow", [11, 30, 100])
@pytest.mark.parametrize("Hq,H,Lq,L,d,cuts", [
    (32, 32, 1024, 1030, 64, [10, 70, 500, 503, 900, 1025]),
    (8, 4, 2200, 2200, 128, [1, 2, 64, 1000, 1001, 2100]),   # the first rows see little
    (1, 1, 256, 131072, 32, [130817, 130900, 131071])])      # split over workgroups
def test_values_that_many_rows_do_not_see(gpu_lib, grow, Hq, H, Lq, L, d, cuts):
    """The same where a tile of values is shared by rows that see it in part."""
    say("kv4 attention of many rows, unseen values 2^%d, Hq%d Lq%d L%d d%d" % (grow, Hq, Lq, L, d))
    assert many_rows(H, Hq // H * Lq, L)
    rng = np.random.default_rng(grow + L + d)
    c = filled(rng, 1, H, L, d)
    for k, cut in enumerate(cuts):
        big = rows(rng, (H, 1, d), "strict_f32") * 2.0 ** (grow * (k + 1) / len(cuts))
        c.put(1, 0, np.array([cut]), big.astype(np.float32))
    Q = rows(rng, (1, Hq, Lq, d), "fast_bf16")
    O, LSE = run(gpu_lib, c, Q, L, 0.1, "fast_bf16")
    check_rows_before(c, Q, O, LSE, L, cuts, 0.1, False, sorted({0, Hq - 1}))


def test_many_rows_before_values_and_zeros(gpu_lib):
    """Rows that see nothing but V = 0 get 0, and rows whose values are tiny theirs,
    whatever comes behind them."""
    say("kv4 attention of many rows, zeros and tiny values first")
    rng = np.random.default_rng(21)
    H, L, d = 32, 1024, 32
    c = filled(rng, 1, H, L, d)
    x = rows(rng, (H, L, d), "strict_f32")
    x[:, :5] = 0
    x[:, 5:30] *= 2.0 ** -60
    c.put(1, 0, np.arange(L), x)
    Q = rows(rng, (1, H, L, d), "fast_bf16")
    O, LSE = run(gpu_lib, c, Q, L, 0.1, "fast_bf16")
    assert not host(O)[0, :, :5].any()
    check_rows_before(c, Q, O, LSE, L, [30], 0.1, False, [0, H - 1])


@pytest.mark.parametrize("cut", [640, 645, 703])
def test_many_rows_before_a_leap(gpu_lib, cut):
    """Values of 2^-70, then one of 2^80, at the start of a tile, within one and at its
    end, where some rows of a wave see the tile and others end before it."""
    say("kv4 attention of many rows before a leap at %d" % cut)
    rng = np.random.default_rng(cut)
    H, Lq, L, d = 32, 1024, 1030, 64
    c = filled(rng, 1, H, L, d)
    x = rows(rng, (H, L, d), "strict_f32") * np.float32(2.0 ** -70)
    for _ in range(2):   # (2^150 is no f32)
        x[:, cut] *= np.float32(2.0 ** 75)
    c.put(1, 0, np.arange(L), x)
    Q = rows(rng, (1, H, Lq, d), "fast_bf16")
    O, LSE = run(gpu_lib, c, Q, L, 0.1, "fast_bf16")
    check_rows_before(c, Q, O, LSE, L, [cut], 0.1, False, [0, H - 1])


# few rows; rows whose weights are recomputed; many rows
FORMS = [("fast_bf16", 1, 3, 70), ("strict_f32", 1, 3, 70), ("fast_bf16", 1, 40, 70),
         ("strict_f32", 1, 40, 70), ("fast_bf16", 32, 64, 8200)]


def one_head(rng, L, d, K=None, V=None):
    """A cache of one head with these rows, or ordinary ones."""
    c = filled(rng, 1, 1, L, d)
    for which, x in ((0, K), (1, V)):
        if x is not None:
            c.put(which, 0, np.arange(L), x.astype(np.float32))
    return c


def check_heads(mg, rng, c, Q, H, scale, contract):
    """Attention with weights over H heads that all hold what c's one does; the first
    and the last two query heads against the reference."""
    import torch
    _, Hq, Lq, d = Q.shape
    L, G, strict = c.dims[2], Hq // H, contract != "fast_bf16"
    whole = ref.Cache(1, H, L, d)
    for which in range(2):
        whole.code[which] = np.repeat(c.code[which], H, 1)
        whole.word[which] = np.repeat(c.word[which], H, 1)
    w0 = rng.random((1, H, L)).astype(np.float32)
    weight = dev(w0)
    O, LSE = mg.attention_forward_kv4(dev(Q, dtype_of(contract)), dev(whole.to_bytes()), H=H, L=L,
                                      causal=True, scale=scale, weight=weight, contract=contract)
    O, LSE, weight = (host(t).astype(np.float64) for t in (O, LSE, weight))
    for h in sorted({0, H - 1}):
        W, tW = np.zeros(L), np.zeros(L)
        for hq in range(h * G, (h + 1) * G):
            rO, rL, P, tO, tL, tP = ref.attention(
                Q[0, hq].astype(np.float64), [x[0, 0] for x in c.code],
                [tuple(p[0, 0] for p in c.group(i)) for i in range(2)], L, Lq, True, scale, strict,
                not strict and many_rows(H, G * Lq, L))
            assert np.all(np.abs(LSE[0, hq] - rL) <= tL), (hq, (np.abs(LSE[0, hq] - rL) / tL).max())
            assert np.all(np.abs(O[0, hq] - rO) <= tO), (hq, (np.abs(O[0, hq] - rO) / tO).max())
            W += P.sum(0)
            tW += tP.sum(0)
        w = w0[0, h].astype(np.float64)
        assert np.all(np.abs(weight[0, h] - (w + W)) <= tW + 2.0 ** -22 * (w + W)), h


@pytest.mark.parametrize("contract,H,Lq,L", FORMS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("q,k,scale", [
    (1e-30, 1e37, 1e-7),             # products of K and codes beyond f32, scores of some units
    (2.0 ** -100, 2.0 ** 123, 2.0 ** -26),   # |scale| max |Q| below the smallest normal
    (2.0 ** -120, 2.0 ** 120, -0.3),
    (2.0 ** 120, 2.0 ** -120, 0.3),
    (1e-5, 1e-35, 1e38),
    (2.0 ** 100, 2.0 ** 120, 0.0),   # scores of 0 all the same
    (0.0, 2.0 ** 124, 2.0 ** 100)])
def test_keys_and_queries_of_any_size(gpu_lib, contract, H, Lq, L, d, q, k, scale):
    """Only the scores have to be in range, not the parts they are made of."""
    say("kv4 attention q %g k %g scale %g d%d %s Lq%d" % (q, k, scale, d, contract, Lq))
    rng = np.random.default_rng(17)
    c = one_head(rng, L, d, K=k * rng.standard_normal((1, L, d)))
    Q = ref.bf16_round((q * rng.standard_normal((1, 2 * H, Lq, d))).astype(np.float32))
    check_heads(gpu_lib, rng, c, Q, H, scale, contract)


@pytest.mark.parametrize("contract,H,Lq,L", FORMS)
def test_queries_of_every_size_over_large_keys(gpu_lib, contract, H, Lq, L):
    """Rows of 1, 2^-60, 2^-100 and 0 beside one another: the small ones' scores are 0."""
    say("kv4 attention, rows of every size %s Lq%d" % (contract, Lq))
    rng = np.random.default_rng(18)
    d = 64
    c = one_head(rng, L, d, K=2.0 ** 122 * rng.standard_normal((1, L, d)))
    Q = ref.bf16_round(rng.standard_normal((1, 2 * H, Lq, d)).astype(np.float32))
    Q[0, :, 0] *= np.float32(2.0 ** -60)
    Q[0, 0, 1] *= np.float32(2.0 ** -100)
    Q[0, 1, 1] = 0
    check_heads(gpu_lib, rng, c, Q, H, 2.0 ** -122, contract)


def test_tiny_values_of_many_tokens(gpu_lib):
    """Equal probabilities of 202,135 tokens whose V is 2^-104 throughout: every sum is
    exact, and O is that value.  (Row tiles enough that tokens are not split.)"""
    import torch
    mg = gpu_lib
    say("kv4 attention of many rows, V of 2^-104")
    n, d, Lq = 202135, 32, 256 * 256
    V = torch.full((1, 1, n, d), 2.0 ** -104, dtype=torch.bfloat16, device="cuda")
    cache = mg.kv4_cache(1, 1, n, d)
    mg.mg_kv4_append(V, V, cache, L=n)
    assert mg.mg_attn_fwd_kv4_workspace_bytes(1, 1, 1, Lq, n, d) == 0
    Q = torch.zeros(1, 1, Lq, d, dtype=torch.bfloat16, device="cuda")
    O, LSE = mg.attention_forward_kv4(Q, cache, H=1, L=n, causal=False, scale=1.0)
    assert bool((O == 2.0 ** -104).all())
    # the logarithm's two ulps and one more for its sum with the maximum
    assert float((LSE.double() - np.log(n)).abs().max()) <= 3 * 2.0 ** -23 * np.log(n)


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("Lq", [4, 24, 200])
def test_strict_weights_of_codes_around_zero(gpu_lib, Lq, d):
    """Keys of codes 8 but for two channels that no query has: every score is 0 exactly,
    a sum of parts less 8 that are 0 each; as scale code + min it is a difference of
    numbers in the thousands, off by a hundredth.  So rows give every token alike."""
    import torch
    mg = gpu_lib
    say("kv4 strict weights, codes around zero Lq%d d%d" % (Lq, d))
    rng = np.random.default_rng(19)
    L = 64
    K = np.zeros((1, 1, L, d), np.float32)
    g = min(d, 64)
    K[..., 0::g], K[..., 1::g] = -8, 7          # scale 1, minimum -8
    c = ref.Cache(1, 1, L, d)
    c.put(0, 0, np.arange(L), K[0])
    c.put(1, 0, np.arange(L), rows(rng, (1, L, d), "strict_f32"))
    assert (c.code[0][..., 2:g] == 8).all() and np.all(c.group(0)[0] == 1)
    Q = np.abs(rows(rng, (1, 1, Lq, d), "strict_f32")) + 0.5
    Q[..., 0::g] = Q[..., 1::g] = 0
    weight = torch.zeros(1, 1, L, device="cuda")
    O, LSE = mg.attention_forward_kv4(dev(Q), dev(c.to_bytes()), H=1, L=L, causal=False, scale=300.0,
                                      weight=weight, contract="strict_f32")
    # a row: LSE's rounding, of a number below 5, twice; sums of Lq probabilities
    tol = (2 * 5 + 4 + Lq) * 2.0 ** -24
    assert np.all(np.abs(host(LSE) - np.log(L)) <= 5 * 2.0 ** -23)
    assert np.all(np.abs(host(weight) * L / Lq - 1) <= tol)


def long_cache(mg, L, d, contract, K, V):
    """L tokens in pieces; K, V: functions of a piece's first token and length to f32
    tensors [n] that all channels have."""
    import torch
    cache, n, dt = mg.kv4_cache(1, 1, L, d), 1 << 21, dtype_of(contract)
    for at in range(0, L, n):
        m = min(n, L - at)
        k, v = (f(at, m).to(dt)[None, None, :, None].expand(1, 1, m, d).contiguous()
                for f in (K, V))
        mg.mg_kv4_append(k, v, cache, dev(np.array([at], np.int32)), L=L, contract=contract)
    return cache


@pytest.mark.parametrize("contract,Lq", [("fast_bf16", 1), ("strict_f32", 3), ("fast_bf16", 256)])
def test_every_token_of_the_longest_sequence(gpu_lib, contract, Lq):
    """2^24 tokens of score 0 whose values are whole numbers below 16: a wave's and a
    workgroup's sums are exact, so what is left are the roundings of joining 64 of
    them, and three blocks of 32 tokens dropped or taken twice would show in LSE."""
    import torch
    mg = gpu_lib
    say("kv4: every one of 2^24 tokens, %s Lq%d" % (contract, Lq))
    L, d = 1 << 24, 32
    torch.manual_seed(20)
    total = []

    def whole(at, m):   # larger ones later, so that a piece's place shows
        v = torch.randint(0, 4, (m,), device="cuda") + 12 * at // L
        total.append(int(v.sum()))
        return v.float()

    cache = long_cache(mg, L, d, contract, lambda at, m: torch.ones(m, device="cuda"), whole)
    Q = torch.zeros(1, 1, Lq, d, dtype=dtype_of(contract), device="cuda")
    O, LSE = mg.attention_forward_kv4(Q, cache, H=1, L=L, causal=False, scale=1.0,
                                      contract=contract)
    mean = sum(total) / L
    tol = 2.0 ** -8 if contract == "fast_bf16" else 2.0 ** -24
    # joining: at most 64 sums, products and the quotient
    assert float((O.double() - mean).abs().max()) <= mean * (tol + 70 * 2.0 ** -24)
    assert float((LSE.double() - 24 * np.log(2)).abs().max()) <= 2 * 2.0 ** -23 * 24 * np.log(2)


def test_sums_of_many_rows_over_many_tokens(gpu_lib):
    """Equal scores whose probabilities are no power of two round the same way at every
    addition, so a chain of sums over all tokens drifts (2^23 of them: LSE by 2^-7).
    Chains have at most 2^18 tokens, of which a lane adds 2^15 sums of four."""
    import torch
    mg = gpu_lib
    say("kv4 attention of many rows, equal scores of 2^23 tokens")
    L, d, Lq, score = 1 << 23, 32, 256 * 256, 0.6180339
    cache = long_cache(mg, L, d, "fast_bf16", lambda at, m: torch.ones(m, device="cuda"),
                       lambda at, m: torch.full((m,), 0.7109375, device="cuda"))
    Q = torch.ones(1, 1, Lq, d, dtype=torch.bfloat16, device="cuda")
    O, LSE = mg.attention_forward_kv4(Q, cache, H=1, L=L, causal=False, scale=score / d)
    sums = 2.0 ** 15 * 2.0 ** -24
    assert float((LSE.double() - (score + np.log(L))).abs().max()) <= sums + 2.0 ** -20
    assert float((O.double() / 0.7109375 - 1).abs().max()) <= 2 * sums + 2.0 ** -8


@pytest.mark.parametrize("Lq", [3, 24])
def test_strict_queries_with_one_large_channel(gpu_lib, Lq):
    """A channel 2^20 above a query's others, whose keys are 0: the others are held within
    2^-39 of it (two f16 parts, of which the second ends at 2^-24 where the largest value
    lies above 2^14), so scores are off by that times the keys beside the reference's
    bound."""
    say("kv4 strict queries with one large channel Lq%d" % Lq)
    rng = np.random.default_rng(22)
    L, d, scale = 200, 64, 0.1
    K = rng.integers(-7, 7, (1, 1, L, d)).astype(np.float32)
    K[..., 0], K[..., 1], K[..., 2] = -8, 7, 0          # scale 1, base 0: exact
    c = one_head(rng, L, d, K=K[0])
    assert np.array_equal(c.rows(0)[0, 0, :L], K[0, 0])
    Q = rng.standard_normal((1, 1, Lq, d)).astype(np.float32)
    Q[..., 2] = 2.0 ** 20
    O, LSE = gpu_lib.attention_forward_kv4(dev(Q), dev(c.to_bytes()), H=1, L=L, causal=True,
                                           scale=scale, contract="strict_f32")
    rO, rL, _, tO, tL, _ = ref.attention(
        Q[0, 0].astype(np.float64), [x[0, 0] for x in c.code],
        [tuple(p[0, 0] for p in c.group(i)) for i in range(2)], L, Lq, True, scale, True)
    score = scale * 2.0 ** (20 - 39) * np.abs(K).sum(-1).max()
    O, LSE = host(O)[0, 0].astype(np.float64), host(LSE)[0, 0].astype(np.float64)
    assert np.all(np.abs(LSE - rL) <= tL + score)
    assert np.all(np.abs(O - rO) <= tO + 2 * score * np.abs(c.rows(1)).max())


@pytest.mark.parametrize("fill", [3e38, -1e30, np.inf, np.nan, 0.0])
@pytest.mark.parametrize("contract,Hq,H,Lq,L", [
    ("fast_bf16", 4, 2, 5, 70), ("strict_f32", 4, 2, 5, 70), ("fast_bf16", 4, 2, 60, 300),
    ("strict_f32", 4, 2, 60, 300), ("fast_bf16", 16, 8, 600, 4000)])
def test_rows_behind_the_last_query_may_hold_anything(gpu_lib, contract, Hq, H, Lq, L, fill):
    """Query rows at and behind q_len have no part in what the others get."""
    import torch
    mg = gpu_lib
    say("kv4 attention, padding of %g %s Lq%d" % (fill, contract, Lq))
    rng = np.random.default_rng(23)
    B, d, dt = 3, 64, dtype_of(contract)
    K, V = (dev(rows(rng, (B, H, L, d), contract), dt) for _ in range(2))
    cache = mg.kv4_cache(B, H, L, d)
    mg.mg_kv4_append(K, V, cache, L=L, contract=contract)
    q_len = [Lq, Lq // 2 + 1, 0]
    Q = dev(rows(rng, (B, Hq, Lq, d), contract), dt)

    def run():
        w = torch.zeros(B, H, L, device="cuda")
        O, LSE = mg.attention_forward_kv4(Q, cache, H=H, L=L, causal=True, scale=0.1, weight=w,
                                          q_len=dev(np.array(q_len, np.int32)), contract=contract)
        return O, LSE, w

    want = run()
    for b, n in enumerate(q_len):
        Q[b, :, n:] = fill
    for a, b in zip(run(), want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("Hq,H,Lq,L,d", [(16, 4, 700, 4000, 64), (6, 2, 1500, 3100, 128)])
def test_many_rows_of_a_padded_batch_before_far_values(gpu_lib, Hq, H, Lq, L, d):
    """Sequences of different length and number of rows, grouped heads: in each a token
    2^70 above the others somewhere among those that only later rows see."""
    mg = gpu_lib
    say("kv4 attention of many rows, a padded batch, far values Hq%d Lq%d d%d" % (Hq, Lq, d))
    key_len, q_len = [L - 7, Lq, Lq + 300, 0], [Lq, Lq, Lq - 90, 5]
    B = len(key_len)
    assert many_rows(B * H, Hq // H * Lq, L)
    rng = np.random.default_rng(24)
    c = filled(rng, B, H, L, d)
    cuts = [n - q + 3 * q // 5 for n, q in zip(key_len, q_len)]
    for b, cut in enumerate(cuts[:3]):
        big = rows(rng, (H, 1, d), "strict_f32") * np.float32(2.0 ** 70)
        c.put(1, b, np.array([cut]), big.astype(np.float32))
    Q = rows(rng, (B, Hq, Lq, d), "fast_bf16")
    ints = lambda x: dev(np.array(x, np.int32))
    O, LSE = mg.attention_forward_kv4(dev(Q, dtype_of("fast_bf16")), dev(c.to_bytes()), H=H, L=L,
                                      causal=True, scale=0.1, key_len=ints(key_len),
                                      q_len=ints(q_len), contract="fast_bf16")
    O, LSE = host(O).astype(np.float64), host(LSE).astype(np.float64)
    for b in range(B):
        n, q = key_len[b], q_len[b]
        assert not O[b, :, q:].any() and np.isneginf(LSE[b, :, q:]).all()
        if n == 0:
            assert not O[b].any() and np.isneginf(LSE[b]).all()
            continue
        for hq in (0, Hq - 1):
            h = hq // (Hq // H)
            done = 0
            for end in (cuts[b], n):
                m = end - (n - q)
                rO, rL, _, tO, tL, _ = ref.attention(
                    Q[b, hq, :m].astype(np.float64), [x[b, h] for x in c.code],
                    [tuple(p[b, h] for p in c.group(i)) for i in range(2)], end, m, True, 0.1,
                    False, True)
                tO = tO + MANY_UNITS * np.abs(c.rows(1)[b, h, :end]).max()
                assert np.all(np.abs(O[b, hq, done:m] - rO[done:]) <= tO[done:]), (b, hq, end)
                assert np.all(np.abs(LSE[b, hq, done:m] - rL[done:]) <= tL[done:]), (b, hq, end)
                done = m
