"""The paged cache on the GPU (mg_paged.h) against the plain 64-bit
implementation in paged_ref.py: tables and slots, rows and bounds written,
attention, selection, attention over the selected pages, and a run of all
together."""
import math

import numpy as np
import pytest

import paged_ref as ref
from gpu_util import say

pytestmark = pytest.mark.gpu


def kind_of(contract):
    return "bf16" if contract == "fast_bf16" else "f32"


def dtype_of(contract):
    import torch
    return torch.bfloat16 if contract == "fast_bf16" else torch.float32


def dev(x, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return t if dtype is None else t.to(dtype)


def ints(x):
    return None if x is None else dev(np.asarray(x, np.int32))


def host(t):
    return t.float().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def rounded(x, contract):
    """What a tensor of the contract's type holds of x, in f32."""
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x, np.float32))
    return t.to(dtype_of(contract)).float().numpy()


def rows(rng, shape, contract):
    return rounded(rng.standard_normal(shape) * np.exp(0.5 * rng.standard_normal(shape[-1])) +
                   0.5 * rng.standard_normal(shape[-1]), contract)


def on_grid(rng, shape):
    """Values whose products and sums are exact in 64 bits, in either type."""
    return (rng.integers(-127, 128, shape) * 2.0 ** rng.integers(-6, 2, shape)).astype(np.float32)


# ---------------------------------------------------------------------- tables --
RESIZE = [
    # B, P, page, N, T, key_len, want, free_count
    (1, 1, 16, 1, 1, [0], [1], 1),
    (3, 4, 16, 12, 64, [0, 15, 16], [1, 17, 48], 9),
    (4, 3, 32, 12, 40, [96, 0, 33, 5], [0, 40, 30, 5], 3),         # one ends, one is cut back
    (3, 4, 16, 6, 64, [16, 0, 15], [32, 64, 16], 1),               # the second waits for pages
    (3, 4, 16, 6, 64, [16, 0, 16], [32, 64, 48], 2),               # the third behind it as well
    (2, 2, 64, 9, 30, [3, 100], [20, 120], 4),                     # the second's rows do not fit
    (3, 2, 16, 9, 100, [30, 3, 0], [40, 33, 20], 4),               # above P * page
    (2, 3, 128, 6, 300, [384, 0], [0, 256], 0),                    # pages taken as they come back
    (4, 2, 256, 9, 50, [-5, 9999, 512, 3], [4, 512, -2, -9], 3),   # clamped
    (2, 2, 16, 4, 9, [0, 0], [4, 5], 99),
    (2, 2, 16, 4, 9, [0, 0], [20, 2 ** 31 - 1], -3),
    (3, 4, 16, 5, 9, [64, 64, 64], [0, 0, 0], 0),                  # more back than N
]


def random_resize(rng, B, P, page, T, most):
    N = B * P
    order = rng.permutation(N).reshape(B, P)
    lens = rng.integers(0, P * page + 1, B) * (rng.random(B) < 0.6)
    held = np.arange(P) < -(-lens // page)[:, None]
    rest = order[~held]
    free = np.concatenate([rest, np.full(N - len(rest), -9)])
    want = np.where(rng.random(B) < 0.2, 0, lens + rng.integers(-3, most + 1, B))
    return (N, lens, want, np.where(held, order, -7), free,
            int(len(rest) * rng.choice([1.0, 0.3])))


def check_resize(mg, page, T, key_len, want, table, free, count, in_place):
    import torch
    B, P = table.shape
    d = [ints(x) for x in (key_len, want, table, free, [count])]
    fill = lambda n: torch.full((n,), -77, dtype=torch.int32, device="cuda")
    new_len, new_count = (d[0], d[4]) if in_place else (fill(B), fill(1))
    slot, offset = fill(T), fill(B + 1)
    mg.mg_paged_resize(*d[:5], new_len, new_count, slot, offset, page=page)
    table, free = np.array(table), np.array(free)
    r_len, r_count, r_slot, r_off = ref.resize(key_len, want, table, free, count, page, T)
    for got, want_, what in ((new_len, r_len, "len"), (offset, r_off, "offset"),
                             (slot, r_slot, "slot"), (d[2], table, "table"), (d[3], free, "free"),
                             (new_count, [r_count], "count")):
        assert np.array_equal(host(got), want_), what


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,P,page,N,T,key_len,want,count", RESIZE)
def test_resize(gpu_lib, B, P, page, N, T, key_len, want, count, in_place):
    say("paged resize B%d P%d page%d T%d" % (B, P, page, T))
    rng = np.random.default_rng(N + T)
    table = rng.integers(0, N, (B, P))
    free = rng.permutation(N)
    check_resize(gpu_lib, page, T, key_len, want, table, free, count, in_place)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,P,page,T,most", [
    (7, 5, 16, 100, 40), (64, 40, 16, 2048, 30), (64, 40, 16, 2049, 60), (300, 9, 32, 5000, 20),
    (1024, 3, 16, 1024, 1), (1025, 3, 16, 1025, 1), (2500, 4, 64, 60000, 200),
    (3, 2000, 128, 400000, 200000)])
def test_resize_many(gpu_lib, B, P, page, T, most, in_place):
    say("paged resize many B%d P%d page%d T%d" % (B, P, page, T))
    N, lens, want, table, free, count = random_resize(np.random.default_rng(B), B, P, page, T, most)
    check_resize(gpu_lib, page, T, lens, want, table, free, count, in_place)


def test_resize_with_entries_outside_the_pool(gpu_lib):
    """Such pages go round and get no slots."""
    say("paged resize bad entries")
    table = np.array([[5, -1, 3], [99, 2, 1]])
    free = np.array([0, -4, 1 << 30, 2, 4, 1])
    check_resize(gpu_lib, 16, 60, [20, 40], [40, 0], table, free, 3, False)
    check_resize(gpu_lib, 16, 60, [0, 0], [33, 20], table, free, 3, False)


# ---------------------------------------------------------------------- append --
APPEND = [
    # H, page, d, N, slots as runs (first slot, rows)
    (1, 16, 32, 1, [(0, 1)]),
    (3, 16, 64, 9, [(5, 1), (16, 1), (100, 1), (143, 1)]),
    (2, 16, 128, 20, [(0, 16), (40, 8), (64, 3), (-1, 2), (100, 12)]),
    (2, 32, 128, 20, [(7, 1), (40, 24), (96, 32), (300, 1), (-1, 5), (9999, 3), (128, 9)]),
    (2, 64, 64, 20, [(3, 61), (128, 64), (640, 2), (-5, 1), (764, 4), (192, 40)]),
    (1, 128, 32, 9, [(17, 111), (128, 128), (400, 100), (-1, 70)]),
    (2, 256, 128, 4, [(10, 246), (256, 256), (512, 1)]),
    (4, 256, 64, 4, [(1, 200), (512, 256)]),
]


def many_runs(rng, page, N, T):
    """Pages in any order, each from some row on, until T rows are there."""
    runs, t = [], 0
    for p in rng.permutation(N):
        first = int(rng.integers(0, page)) if rng.random() < 0.3 else 0
        n = int(min(page - first if rng.random() < 0.8 else rng.integers(1, page - first + 1), T - t))
        if n <= 0:
            break
        runs.append((int(p) * page + first, n))
        t += n
    return runs


def slots_of(runs):
    return np.concatenate([np.arange(s, s + n) if s >= 0 else np.full(n, s) for s, n in runs])


def check_append(mg, rng, H, page, d, N, slot, contract, with_bounds=True, K=None):
    kind, dt, T = kind_of(contract), dtype_of(contract), len(slot)
    pages = [s // page for k, s in enumerate(slot) if 0 <= s < N * page and
             not (k and s % page and slot[k - 1] == s - 1)]
    assert len(set(pages)) == len(pages)   # what the call asks of its slots
    K = rows(rng, (T, H, d), contract) if K is None else K
    V = rows(rng, (T, H, d), contract)
    Kp, Vp = (rows(rng, (N, H, page, d), contract) for _ in range(2))
    bounds = rows(rng, (N, H, 2, d), contract) if with_bounds else None
    g = [dev(x, dt) for x in (K, V, Kp, Vp)]
    gb = dev(bounds, dt) if with_bounds else None
    mg.mg_paged_append(*g, ints(slot), gb, contract=contract)
    ref.append(K, V, Kp, Vp, bounds, slot, kind)
    assert np.array_equal(host(g[2]), Kp, equal_nan=True)
    assert np.array_equal(host(g[3]), Vp, equal_nan=True)
    if with_bounds:
        assert np.array_equal(host(gb), bounds)


@pytest.mark.parametrize("contract", ["fast_bf16", "strict_f32", "accelerated"])
@pytest.mark.parametrize("H,page,d,N,runs", APPEND)
def test_append(gpu_lib, H, page, d, N, runs, contract):
    say("paged append H%d page%d d%d %s" % (H, page, d, contract))
    check_append(gpu_lib, np.random.default_rng(page + d), H, page, d, N, slots_of(runs), contract)


@pytest.mark.parametrize("contract", ["fast_bf16", "strict_f32"])
@pytest.mark.parametrize("H,page,d,T", [(8, 16, 128, 2500), (8, 64, 128, 2500), (4, 128, 64, 5000),
                                        (2, 256, 32, 9000), (1, 32, 32, 17000), (5, 16, 64, 3500)])
def test_append_many(gpu_lib, H, page, d, T, contract):
    say("paged append many H%d page%d d%d T%d %s" % (H, page, d, T, contract))
    rng = np.random.default_rng(T)
    N = T // page * 2 + 2
    check_append(gpu_lib, rng, H, page, d, N, slots_of(many_runs(rng, page, N, T)), contract)


def test_append_without_bounds(gpu_lib):
    say("paged append without bounds")
    check_append(gpu_lib, np.random.default_rng(1), 2, 16, 64, 9, slots_of([(5, 11), (32, 3)]),
                 "fast_bf16", with_bounds=False)


@pytest.mark.parametrize("contract", ["fast_bf16", "strict_f32"])
def test_append_special_values(gpu_lib, contract):
    """NaN is left out of bounds, infinities count as the largest value."""
    say("paged append special values %s" % contract)
    rng = np.random.default_rng(2)
    slot = slots_of([(0, 16), (84, 3), (176, 1), (192, 40)])
    K = rows(rng, (len(slot), 2, 64), contract)
    K[::3, :, 5] = np.nan
    K[:, :, 6] = np.nan
    K[::2, :, 7], K[1::2, :, 7] = np.inf, -np.inf
    K[:, :, 8], K[:, :, 9] = -np.inf, 0.0
    check_append(gpu_lib, rng, 2, 64, 64, 4, slot, contract, K=K)


# ------------------------------------------------------------------- attention --
ATTN = [
    # B, Hq, H, Lq, d, page, P, key_len, q_len, causal
    (1, 1, 1, 1, 32, 16, 1, [1], None, True),
    (1, 4, 4, 1, 64, 16, 16, [256], None, True),
    (2, 6, 2, 1, 128, 32, 2, [31, 1], None, False),
    (3, 8, 1, 1, 128, 64, 12, [0, 700, 33], None, True),
    (2, 4, 2, 3, 64, 16, 8, [100, 2], [3, 3], True),       # a first row that sees nothing
    (2, 6, 3, 7, 32, 128, 2, [201, 64], [7, 2], True),
    (2, 2, 2, 5, 128, 16, 5, [40, 64], [5, 0], False),
    (1, 3, 1, 20, 64, 32, 11, [333], [18], True),
    (1, 24, 1, 2, 128, 256, 3, [555], None, True),         # 48 rows a cache head
    (2, 8, 8, 1, 64, 16, 130, [2000, 77], None, True),
    (1, 8, 2, 2, 128, 16, 400, [4999], None, True),        # many units of one sequence
    (5, 4, 2, 1, 128, 16, 70, [1100, 3, 0, 640, 64], None, True),
    (1, 8, 2, 40, 64, 16, 40, [610], [37], True),          # 160 rows a cache head
    (2, 80, 1, 1, 32, 64, 12, [700, 90], None, True),
    (70, 8, 4, 1, 64, 16, 40, [(37 * b) % 600 for b in range(70)], None, True),   # by lengths
    (3, 4, 4, 2, 32, 64, 900, [50000, 57600, 1], None, True),
    (2, 16, 1, 1, 128, 64, 2000, [90000, 128000], None, True),
    (700, 2, 1, 1, 32, 16, 700, [(b * 7919) % 90 if b != 333 else 11000 for b in range(700)], None,
     True),
    (65, 8, 8, 3, 64, 64, 40, [2560 - 30 * b for b in range(65)], None, True),
    (256, 2, 1, 1, 32, 16, 130, [(b * 7919) % 2080 for b in range(256)], None, True),
    (257, 2, 1, 1, 32, 16, 130, [(b * 7919) % 2080 for b in range(257)], None, True),
    (130, 2, 2, 1, 32, 32, 33, [1056 - 8 * b for b in range(130)], None, False),
]


def table_of(rng, B, P, page, key_len):
    """A table of distinct pages, entries behind a sequence's last one wild."""
    need = [ref.pages(min(max(n, 0), P * page), page) for n in key_len]
    N = sum(need) + 2
    order = rng.permutation(N)
    table = rng.choice([-1, 1 << 30, N, 0], (B, P))
    at = 0
    for b, m in enumerate(need):
        table[b, :m] = order[at:at + m]
        at += m
    return N, table


def pooled(rng, N, H, page, d, contract):
    return [rows(rng, (N, H, page, d), contract) for _ in range(2)]


def check_attention(mg, Q, Kp, Vp, table, key_len, q_len, causal, scale, contract, index=None,
                    sequences=None):
    import torch
    B, Hq, Lq, d = Q.shape
    N, H, page, _ = Kp.shape
    P, kind, dt = table.shape[1], kind_of(contract), dtype_of(contract)
    O = torch.full(Q.shape, math.nan, dtype=dt, device="cuda")
    LSE = torch.full(Q.shape[:3], math.nan, device="cuda")
    kw = dict(causal=causal, scale=scale, contract=contract)
    args = (dev(Q, dt), dev(Kp, dt), dev(Vp, dt), ints(table), ints(key_len))
    if index is None:
        mg.mg_attn_fwd_paged(*args, O, LSE, ints(q_len), **kw)
    else:
        mg.mg_attn_fwd_paged_sparse(*args, ints(index), O, LSE, ints(q_len), **kw)
    gO, gL = host(O).astype(np.float64), host(LSE).astype(np.float64)
    for b in range(B) if sequences is None else sequences:
        n = min(max(int(key_len[b]), 0), P * page)
        r = Lq if q_len is None else min(max(int(q_len[b]), 0), Lq)
        for h in range(H):
            for i in range(Lq):
                sees = ref.limit(n, r, i, causal)
                if index is None:
                    ids = table[b, np.arange(sees) // page]
                    ok = (ids >= 0) & (ids < N)
                    at, row = ids[ok], (np.arange(sees) % page)[ok]
                else:
                    tokens = ref.listed(index[b, h, i], table[b], page, sees, P, N)
                    at, row = [t[1] for t in tokens], [t[2] for t in tokens]
                k, v = (x[at, h, row].reshape(-1, d) for x in (Kp, Vp))
                for hq in range(h * (Hq // H), (h + 1) * (Hq // H)):
                    rO, rL, tO, tL = ref.attention(Q[b, hq, i], k, v, scale, kind)
                    where = (b, hq, i)
                    if np.isneginf(rL):
                        assert np.isneginf(gL[where]) and np.all(gO[where] == 0), where
                        continue
                    assert abs(gL[where] - rL) <= tL, (where, gL[where], rL, tL)
                    off = np.abs(gO[where] - rO)
                    assert np.all(off <= tO), (where, (off / tO).max())


@pytest.mark.parametrize("contract", ["fast_bf16", "strict_f32"])
@pytest.mark.parametrize("B,Hq,H,Lq,d,page,P,key_len,q_len,causal", ATTN)
def test_attention(gpu_lib, B, Hq, H, Lq, d, page, P, key_len, q_len, causal, contract):
    say("paged attention B%d Hq%d H%d Lq%d d%d page%d P%d %s" % (B, Hq, H, Lq, d, page, P, contract))
    rng = np.random.default_rng(B * 1000 + P)
    N, table = table_of(rng, B, P, page, key_len)
    Kp, Vp = pooled(rng, N, H, page, d, contract)
    Q = rows(rng, (B, Hq, Lq, d), contract)
    check_attention(gpu_lib, Q, Kp, Vp, table, key_len, q_len, causal, d ** -0.5, contract)


@pytest.mark.parametrize("contract", ["fast_bf16", "strict_f32"])
@pytest.mark.parametrize("sparse", [False, True])
def test_long_units(gpu_lib, contract, sparse):
    """Units of several thousand tokens in pages of 16 (two sequences are checked)."""
    say("paged attention long units %s sparse %s" % (contract, sparse))
    rng = np.random.default_rng(12)
    B, H, d, page, N = 12, 16, 128, 16, 60
    P = 1400 if sparse else 2600
    key_len = [P * page - 5 - (b % 3) for b in range(B)]
    table = rng.integers(0, N, (B, P))
    Kp, Vp = pooled(rng, N, H, page, d, contract)
    Q = rows(rng, (B, H, 1, d), contract)
    index = None
    if sparse:
        B = 64
        table, key_len = np.tile(table, (6, 1))[:B], (key_len * 6)[:B]
        Q = np.tile(Q, (6, 1, 1, 1))[:B]
        index = np.sort(rng.permuted(np.tile(np.arange(P), (B, H, 1, 1)), axis=3)[..., :301], 3)
    check_attention(gpu_lib, Q, Kp, Vp, table, key_len, None, True, d ** -0.5, contract, index,
                    sequences=[0, 11])


@pytest.mark.parametrize("contract", ["fast_bf16", "strict_f32"])
def test_infinite_scores(gpu_lib, contract):
    """Tokens whose score is -inf count as ones with no weight."""
    say("paged attention infinite scores %s" % contract)
    rng = np.random.default_rng(13)
    N, table = table_of(rng, 1, 6, 16, [90])
    Kp, Vp = pooled(rng, N, 1, 16, 64, contract)
    Q = np.abs(rows(rng, (1, 3, 1, 64), contract))
    whole = Kp.copy()
    for j in (0, 17, 50, 89):
        Kp[table[0, j // 16], 0, j % 16, 5] = -np.inf
        whole[table[0, j // 16], 0, j % 16] = -60 / Q.min((0, 1, 2))   # as good as nothing
    for scale in (0.125, 0.1):
        out = [gpu_lib.attention_forward_paged(dev(Q, dtype_of(contract)), dev(k, dtype_of(contract)),
                                               dev(Vp, dtype_of(contract)), ints(table), ints([90]),
                                               causal=True, scale=scale) for k in (Kp, whole)]
        # (exp(-60 * 64 / 10) is 0 in f32: the same sums)
        for a, b in zip(*out):
            assert np.array_equal(host(a), host(b))


def test_accelerated_gives_the_strict_results(gpu_lib):
    import torch
    say("paged attention accelerated")
    rng = np.random.default_rng(9)
    N, table = table_of(rng, 2, 9, 32, [250, 31])
    Kp, Vp = (dev(x) for x in pooled(rng, N, 2, 32, 64, "strict_f32"))
    Q = dev(rows(rng, (2, 4, 1, 64), "strict_f32"))
    a, b = (gpu_lib.attention_forward_paged(Q, Kp, Vp, ints(table), ints([250, 31]), causal=True,
                                            scale=0.1, contract=c)
            for c in ("strict_f32", "accelerated"))
    assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("contract", ["fast_bf16", "strict_f32"])
@pytest.mark.parametrize("scale", [-0.3, 0.0, 30.0])
def test_scales(gpu_lib, scale, contract):
    say("paged attention scale %g %s" % (scale, contract))
    rng = np.random.default_rng(11)
    N, table = table_of(rng, 2, 20, 16, [300, 47])
    Kp, Vp = pooled(rng, N, 2, 16, 64, contract)
    check_attention(gpu_lib, rows(rng, (2, 4, 2, 64), contract), Kp, Vp, table, [300, 47], None, True,
                    scale, contract)


@pytest.mark.parametrize("sparse", [False, True])
@pytest.mark.parametrize("contract", ["fast_bf16", "strict_f32"])
@pytest.mark.parametrize("d,page", [(32, 16), (64, 32), (128, 16), (128, 64)])
def test_what_a_row_does_not_see_has_no_part_in_it(gpu_lib, d, page, contract, sparse):
    """Infinities and NaN behind the sequence, behind the causal mask of some rows,
    in pages that no sequence holds, in query rows behind q_len; then a row that
    sees them."""
    import torch
    say("paged attention masked specials d%d page%d %s" % (d, page, contract))
    rng = np.random.default_rng(d)
    B, Hq, H, Lq, P = 3, 6, 2, 5, 12
    key_len, q_len = [150, 33, 4], [5, 3, 5]
    N, table = table_of(rng, B, P, page, key_len)
    Kp, Vp = pooled(rng, N, H, page, d, contract)
    Q = rows(rng, (B, Hq, Lq, d), contract)
    clean = [x.copy() for x in (Kp, Vp, Q)]
    held = np.zeros((N, page), bool)
    for b, n in enumerate(key_len):
        j = np.arange(n)
        held[table[b, j // page], j % page] = True
    for x in (Kp, Vp):
        x[~held[:, None, :].repeat(H, 1)] = rng.choice([np.nan, np.inf, -np.inf])
    Q[1, :, 3:] = np.nan
    for b, n in enumerate(key_len):   # the last two tokens, which the first rows do not see
        for j in (n - 2, n - 1):
            at, row = table[b, j // page], j % page
            Kp[at, :, row], Vp[at, :, row] = np.nan, np.inf
            Vp[at, 0, row, ::3] = np.nan
            Vp[at, 1, row, ::2] = -np.inf
    index = None
    if sparse:
        index = np.tile(np.concatenate([np.arange(P), [-1]]), (B, H, Lq, 1)).astype(np.int64)
    out = []
    for k, v, q in ((Kp, Vp, Q), clean):
        dt = dtype_of(contract)
        O = torch.full(Q.shape, 9.0, dtype=dt, device="cuda")
        LSE = torch.full(Q.shape[:3], 9.0, device="cuda")
        args = (dev(q, dt), dev(k, dt), dev(v, dt), ints(table), ints(key_len))
        kw = dict(causal=True, scale=0.2, contract=contract)
        if sparse:
            gpu_lib.mg_attn_fwd_paged_sparse(*args, ints(index), O, LSE, ints(q_len), **kw)
        else:
            gpu_lib.mg_attn_fwd_paged(*args, O, LSE, ints(q_len), **kw)
        out.append((host(O), host(LSE)))
    for b in range(B):
        unseen = max(q_len[b] - 2, 0)   # rows that see neither of the two
        for x, y in zip(*out):
            assert np.array_equal(x[b, :, :unseen], y[b, :, :unseen]), b
            assert np.array_equal(x[b, :, q_len[b]:], y[b, :, q_len[b]:]), b
            assert np.isnan(x[b, :, q_len[b] - 1]).any(), b
    check_attention(gpu_lib, clean[2], clean[0], clean[1], table, key_len, q_len, True, 0.2, contract,
                    index)


@pytest.mark.parametrize("contract", ["fast_bf16", "strict_f32"])
def test_infinite_values_reach_the_rows_that_see_them_only(gpu_lib, contract):
    """V infinite in one channel of the last token, K finite: rows before stay
    finite, the last one is infinite there and right elsewhere."""
    say("paged attention infinite value %s" % contract)
    rng = np.random.default_rng(4)
    d, page, n = 64, 16, 70
    N, table = table_of(rng, 1, 5, page, [n])
    Kp, Vp = pooled(rng, N, 1, page, d, contract)
    Q = rows(rng, (1, 2, 4, d), contract)
    Vp[table[0, (n - 1) // page], 0, (n - 1) % page, 7] = np.inf
    O, LSE = gpu_lib.attention_forward_paged(dev(Q, dtype_of(contract)), dev(Kp, dtype_of(contract)),
                                             dev(Vp, dtype_of(contract)), ints(table), ints([n]),
                                             causal=True, scale=0.1)
    O = host(O)
    assert np.isfinite(O[0, :, :3]).all() and np.isposinf(O[0, :, 3, 7]).all()
    assert np.isfinite(np.delete(O[0, :, 3], 7, -1)).all()
    Vp[table[0, (n - 1) // page], 0, (n - 1) % page, 7] = 0.0
    check_attention(gpu_lib, Q[:, :, :], Kp, Vp, table, [n], None, True, 0.1, contract)


@pytest.mark.parametrize("contract", ["fast_bf16", "strict_f32"])
def test_entries_outside_the_pool_and_lengths_outside_the_table(gpu_lib, contract):
    say("paged attention bad entries %s" % contract)
    rng = np.random.default_rng(5)
    N, P, page, d = 6, 5, 16, 64
    table = np.array([[0, -1, 3, 6, 1], [1 << 30, 2, 2, 0, -5], [-1, 99, -2, 7, 6]])
    Kp, Vp = pooled(rng, N, 2, page, d, contract)
    Q = rows(rng, (3, 4, 2, d), contract)
    for key_len in ([80, 75, 80], [2 ** 31 - 1, 1000, -7]):
        check_attention(gpu_lib, Q, Kp, Vp, table, key_len, None, True, 0.125, contract)


@pytest.mark.parametrize("contract", ["fast_bf16", "strict_f32"])
def test_sequences_that_share_pages(gpu_lib, contract):
    say("paged attention shared pages %s" % contract)
    rng = np.random.default_rng(6)
    Kp, Vp = pooled(rng, 9, 2, 32, 128, contract)
    table = np.array([[4, 2, 7, 1], [4, 2, 0, 8], [4, 4, 4, 4]])
    check_attention(gpu_lib, rows(rng, (3, 4, 1, 128), contract), Kp, Vp, table, [128, 100, 97], None,
                    True, 0.09, contract)


# ------------------------------------------------------------------- selection --
SELECT = [
    # B, Hq, H, Lq, d, page, P, key_len, q_len, causal, keep, first, recent
    (1, 1, 1, 1, 32, 16, 1, [9], None, True, 1, 0, 0),
    (1, 1, 1, 1, 32, 16, 9, [140], None, True, 1, 0, 1),
    (2, 4, 2, 1, 64, 16, 40, [640, 100], None, True, 8, 1, 2),
    (3, 8, 1, 1, 128, 32, 70, [0, 2240, 257], None, True, 9, 0, 0),
    (2, 6, 2, 4, 64, 64, 33, [2100, 300], [4, 2], True, 6, 2, 1),
    (1, 10, 2, 7, 32, 16, 50, [790], None, False, 10, 3, 3),
    (1, 40, 2, 3, 128, 16, 30, [478], None, True, 11, 1, 1),     # 20 heads a group
    (2, 8, 8, 1, 128, 16, 1030, [16480, 16000], None, True, 200, 1, 4),
    (1, 4, 1, 1, 32, 16, 5000, [80000], None, True, 1234, 0, 0),
    (1, 2, 1, 1, 64, 256, 20, [5000], None, True, 5, 3, 2),      # nothing left to choose
    (2, 4, 2, 2, 64, 16, 20, [320, 17], None, True, 40, 1, 1),   # room for more than there are
    (40, 2, 2, 1, 32, 16, 64, [25 * b for b in range(40)], None, True, 16, 1, 1),
    (1, 16, 1, 2, 64, 16, 1024, [16384], None, True, 300, 1, 1),
    (2, 12, 2, 5, 128, 32, 1100, [35200, 9000], [5, 3], True, 77, 2, 2),
    (1, 3, 1, 3, 32, 16, 1500, [24000], None, True, 800, 0, 1),
]


def reference_pages(Q, bounds, table, key_len, q_len, causal, page, keep, first, recent):
    B, Hq, Lq, _ = Q.shape
    H, P = bounds.shape[1], table.shape[1]
    out = np.full((B, H, Lq, keep), -1)
    for b in range(B):
        n = min(max(int(key_len[b]), 0), P * page)
        r = Lq if q_len is None else min(max(int(q_len[b]), 0), Lq)
        for h in range(H):
            for i in range(Lq):
                q = Q[b, h * (Hq // H):(h + 1) * (Hq // H), i]
                out[b, h, i] = ref.select(q, bounds[:, h], table[b],
                                          ref.pages(ref.limit(n, r, i, causal), page), keep, first,
                                          recent)
    return out


def chosen(mg, Q, bounds, table, key_len, q_len, causal, page, keep, first, recent, contract):
    import torch
    B, _, Lq, _ = Q.shape
    index = torch.full((B, bounds.shape[1], Lq, keep), -77, dtype=torch.int32, device="cuda")
    mg.mg_paged_select(dev(Q, dtype_of(contract)), dev(bounds, dtype_of(contract)), ints(table),
                       ints(key_len), index, ints(q_len), page=page, causal=causal, first=first,
                       recent=recent, contract=contract)
    return host(index)


@pytest.mark.parametrize("contract", ["fast_bf16", "strict_f32", "accelerated"])
@pytest.mark.parametrize("B,Hq,H,Lq,d,page,P,key_len,q_len,causal,keep,first,recent", SELECT)
def test_select(gpu_lib, B, Hq, H, Lq, d, page, P, key_len, q_len, causal, keep, first, recent,
                contract):
    say("paged select B%d Hq%d H%d Lq%d d%d page%d P%d keep%d %s"
        % (B, Hq, H, Lq, d, page, P, keep, contract))
    rng = np.random.default_rng(P + keep)
    N, table = table_of(rng, B, P, page, key_len)
    lo, hi = np.sort(on_grid(rng, (2, N, H, d)), 0)
    bounds = np.stack([lo, hi], 2)
    Q = on_grid(rng, (B, Hq, Lq, d))
    want = reference_pages(Q, bounds, table, key_len, q_len, causal, page, keep, first, recent)
    got = chosen(gpu_lib, Q, bounds, table, key_len, q_len, causal, page, keep, first, recent, contract)
    assert np.array_equal(got, want)


def test_select_special_scores(gpu_lib):
    """Equal scores go to the lower index, both zeros are one score, NaN is lowest,
    entries outside the pool count as NaN, infinite bounds."""
    say("paged select special scores")
    rng = np.random.default_rng(3)
    d, page, P, N = 32, 16, 200, 200
    for seed in range(4):
        bounds = np.sort(rng.integers(-1, 2, (2, N, 1, d)).astype(np.float32), 0)
        Q = rng.integers(-1, 2, (1, 2, 1, d)).astype(np.float32)
        if seed % 2:
            Q[:, :, :, 3:] = 0
        lo, hi = bounds
        lo[5:50:7, :, 0], hi[3:60:5, :, 1] = np.nan, np.inf
        lo[8:90:9, :, 2] = -np.inf
        table = rng.permutation(N)[None].copy()
        table[0, 17::31] = -1
        table[0, 40] = N
        both = np.stack([lo, hi], 2)
        for keep, first, recent in ((20, 0, 0), (150, 2, 3), (196, 0, 1)):
            want = reference_pages(Q, both, table, [P * page], None, True, page, keep, first, recent)
            got = chosen(gpu_lib, Q, both, table, [P * page], None, True, page, keep, first, recent,
                         "strict_f32")
            assert np.array_equal(got, want), (seed, keep)


# ---------------------------------------------------------- the selected pages --
SPARSE = [
    # B, Hq, H, Lq, d, page, P, key_len, q_len, keep
    (1, 1, 1, 1, 32, 16, 1, [3], None, 1),
    (2, 4, 2, 1, 64, 16, 40, [640, 90], None, 7),
    (2, 8, 2, 1, 128, 32, 50, [1600, 33], None, 30),
    (1, 6, 3, 4, 64, 64, 30, [1900], [3], 5),
    (2, 4, 1, 2, 128, 16, 300, [4700, 0], None, 129),
    (1, 40, 2, 1, 32, 16, 60, [950], None, 33),
    (1, 4, 1, 1, 128, 64, 200, [12700], None, 101),
    (3, 2, 2, 1, 64, 256, 20, [5000, 256, 257], None, 9),
    (1, 2, 1, 3, 64, 128, 70, [8900], None, 70),
]


@pytest.mark.parametrize("contract", ["fast_bf16", "strict_f32"])
@pytest.mark.parametrize("B,Hq,H,Lq,d,page,P,key_len,q_len,keep", SPARSE)
def test_attention_over_listed_pages(gpu_lib, B, Hq, H, Lq, d, page, P, key_len, q_len, keep,
                                     contract):
    say("paged sparse B%d Hq%d H%d Lq%d d%d page%d P%d keep%d %s"
        % (B, Hq, H, Lq, d, page, P, keep, contract))
    rng = np.random.default_rng(P + keep)
    N, table = table_of(rng, B, P, page, key_len)
    Kp, Vp = pooled(rng, N, H, page, d, contract)
    index = np.full((B, H, Lq, keep), -1)
    for at in np.ndindex(B, H, Lq):
        some = np.sort(rng.permutation(P)[:min(keep, P)])   # behind the sequence's end as well
        index[at][:len(some)] = some
    check_attention(gpu_lib, rows(rng, (B, Hq, Lq, d), contract), Kp, Vp, table, key_len, q_len, True,
                    d ** -0.5, contract, index)


def test_lists_that_repeat_or_reach_outside(gpu_lib):
    say("paged sparse odd lists")
    rng = np.random.default_rng(8)
    page, P, d = 16, 12, 64
    N, table = table_of(rng, 1, P, page, [190])
    Kp, Vp = pooled(rng, N, 1, page, d, "strict_f32")
    Q = rows(rng, (1, 2, 1, d), "strict_f32")
    for index in ([3, 3, 3, 7, 7, -1], [-1, 2, -1, 5, 99, 100], [5, 4, 6, 2, 8, 8],
                  [-1, -1, -1, -1, -1, -1], [2 ** 31 - 1, 3, -2 ** 31, 4, 11, 12],
                  [12, 13, 14, 15, 16, 17]):
        check_attention(gpu_lib, Q, Kp, Vp, table, [190], None, True, 0.125, "strict_f32",
                        np.array(index).reshape(1, 1, 1, 6))


@pytest.mark.parametrize("contract", ["fast_bf16", "strict_f32"])
def test_all_pages_listed_is_the_whole_attention(gpu_lib, contract):
    say("paged sparse all listed %s" % contract)
    rng = np.random.default_rng(10)
    N, table = table_of(rng, 2, 20, 32, [600, 41])
    Kp, Vp = pooled(rng, N, 2, 32, 128, contract)
    Q = rows(rng, (2, 4, 3, 128), contract)
    index = np.tile(np.arange(20), (2, 2, 3, 1))
    check_attention(gpu_lib, Q, Kp, Vp, table, [600, 41], None, True, 0.09, contract, index)


# --------------------------------------------------------------- all together --
@pytest.mark.parametrize("contract", ["fast_bf16", "strict_f32"])
@pytest.mark.parametrize("page", [16, 64])
def test_a_served_batch(gpu_lib, page, contract):
    """Prompts come in, tokens follow, a sequence ends and another takes its place;
    at every step rows are written through the slots, and attention over all and
    over selected pages is checked."""
    import torch
    mg = gpu_lib
    say("paged served batch page%d %s" % (page, contract))
    rng = np.random.default_rng(page)
    B, Hq, H, d, P, N = 3, 4, 2, 64, 8, 20
    kind, dt = kind_of(contract), dtype_of(contract)
    Kp, Vp, bounds = mg.paged_cache(N, H, page, d, contract)
    for t in (Kp, Vp, bounds):
        t.fill_(math.nan)
    table, free = ints(np.full((B, P), -1)), ints(rng.permutation(N))
    length, count = ints([0] * B), ints([N])
    hK, hV = (np.full((N, H, page, d), np.nan, np.float32) for _ in range(2))
    hb = np.full((N, H, 2, d), np.nan, np.float32)
    now = np.zeros(B, int)
    for want in ([page + 5, 0, 3 * page], [page + 6, 2 * page, 3 * page + 1],
                 [page + 7, 2 * page + 1, 0], [page + 8, 2 * page - 2, 7 * page + 3],
                 [2 * page, 2 * page + 5, 7 * page + 4]):
        T = max(int(np.maximum(np.array(want) - now, 0).sum()), 1)
        slot, offset = ints([0] * T), ints([0] * (B + 1))
        mg.mg_paged_resize(length, ints(want), table, free, count, length, count, slot, offset,
                           page=page)
        assert np.array_equal(host(length), want)
        K, V = (rows(rng, (T, H, d), contract) for _ in range(2))
        mg.mg_paged_append(dev(K, dt), dev(V, dt), Kp, Vp, slot, bounds, contract=contract)
        ref.append(K, V, hK, hV, hb, host(slot), kind)
        assert np.array_equal(host(bounds), hb, equal_nan=True)
        now = np.array(want)
        Q = on_grid(rng, (B, Hq, 1, d)) / 64
        Q = rounded(Q, contract)
        check_attention(mg, Q, hK, hV, host(table), want, None, True, 0.125, contract)
        # (the pools hold NaN where nothing was written)
        assert np.array_equal(host(Kp), hK, equal_nan=True)
        index = torch.full((B, H, 1, 3), -77, dtype=torch.int32, device="cuda")
        mg.mg_paged_select(dev(Q, dt), bounds, table, length, index, page=page, causal=True, first=1,
                           recent=1, contract=contract)
        O, LSE = mg.attention_forward_paged(dev(Q, dt), Kp, Vp, table, length, causal=True,
                                            scale=0.125, bounds=bounds, keep=3, first=1, recent=1)
        O2, LSE2 = torch.empty_like(O), torch.empty_like(LSE)
        mg.mg_attn_fwd_paged_sparse(dev(Q, dt), Kp, Vp, table, length, index, O2, LSE2, causal=True,
                                    scale=0.125, contract=contract)
        assert torch.equal(O, O2) and torch.equal(LSE, LSE2)
        check_attention(mg, Q, hK, hV, host(table), want, None, True, 0.125, contract, host(index))
