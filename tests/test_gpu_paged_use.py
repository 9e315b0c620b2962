"""How a program uses the paged cache: inside guarded buffers, captured into a
graph, on several streams and devices, with pools beyond 4 GiB, many sequences
and long ones; and what its entry points refuse."""
import math

import numpy as np
import pytest

import paged_ref as ref
from gpu_util import say
from test_gpu_kv4_use import GUARD, guarded, ints, same

pytestmark = pytest.mark.gpu


def randn(rng, *shape, dtype=None, device="cuda"):
    import torch
    t = torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(device)
    return t.to(dtype or torch.bfloat16)


class Session:
    """A batch and its buffers: prompts in, a step of Lq tokens, attention over all
    and over selected pages."""

    def __init__(self, mg, seed, B=3, Hq=8, H=2, page=16, d=64, n=200, Lq=1, room=400, keep=5,
                 contract="fast_bf16", device="cuda"):
        import torch
        rng = np.random.default_rng(seed)
        self.mg, self.page, self.contract, self.B = mg, page, contract, B
        elem = torch.bfloat16 if contract == "fast_bf16" else torch.float32
        P = ref.pages(room, page)
        N = B * P + 2
        self.prompt = rng.integers(max(1, n // 3), n + 1, B)
        i32 = dict(dtype=torch.int32, device=device)
        self.want = [torch.tensor(self.prompt, **i32), torch.tensor(self.prompt + Lq, **i32)]
        self.T = [B * n, B * Lq]
        self.rows = [[randn(rng, T, H, d, dtype=elem, device=device) for _ in range(2)]
                     for T in self.T]
        self.Q = randn(rng, B, Hq, Lq, d, dtype=elem, device=device)
        self.Kp, self.Vp, self.bounds = mg.paged_cache(N, H, page, d, contract, device=device)
        self.table = torch.empty(B, P, **i32)
        self.start = torch.tensor(rng.permutation(N), **i32)
        self.free = self.start.clone()
        self.count, self.length = torch.empty(1, **i32), torch.empty(B, **i32)
        self.slot = [torch.empty(T, **i32) for T in self.T]
        self.offset = torch.empty(B + 1, **i32)
        self.index = torch.empty(B, H, Lq, keep, **i32)
        self.O, self.O2 = torch.empty_like(self.Q), torch.empty_like(self.Q)
        self.LSE, self.LSE2 = (torch.empty(B, Hq, Lq, device=device) for _ in range(2))
        sizes = (B, Hq, H, Lq, d, page)
        need = max(mg.mg_paged_resize_workspace_bytes(B, max(self.T)),
                   mg.mg_attn_fwd_paged_workspace_bytes(*sizes, P, contract),
                   mg.mg_paged_select_workspace_bytes(*sizes, P, contract),
                   mg.mg_attn_fwd_paged_sparse_workspace_bytes(*sizes, keep, contract), 1)
        self.ws = torch.empty(need, dtype=torch.uint8, device=device)   # one for all calls

    def reset(self):
        self.free.copy_(self.start)
        self.count.fill_(self.free.numel())
        self.length.zero_()
        self.table.fill_(-1)
        for t in (self.Kp, self.Vp, self.bounds, self.O, self.O2, self.LSE, self.LSE2):
            t.fill_(math.nan)
        self.index.zero_()
        self.ws.fill_(0xff)

    def run(self, stream=None, workspace=True):
        mg, ws = self.mg, self.ws if workspace else None
        kw = dict(contract=self.contract, stream=stream)
        for k in range(2):
            mg.mg_paged_resize(self.length, self.want[k], self.table, self.free, self.count,
                               self.length, self.count, self.slot[k], self.offset, page=self.page,
                               workspace=ws, stream=stream)
            mg.mg_paged_append(*self.rows[k], self.Kp, self.Vp, self.slot[k], self.bounds, **kw)
        kw.update(causal=True, workspace=ws)
        mg.mg_attn_fwd_paged(self.Q, self.Kp, self.Vp, self.table, self.length, self.O, self.LSE,
                             scale=0.125, **kw)
        mg.mg_paged_select(self.Q, self.bounds, self.table, self.length, self.index, page=self.page,
                           first=1, recent=1, **kw)
        mg.mg_attn_fwd_paged_sparse(self.Q, self.Kp, self.Vp, self.table, self.length, self.index,
                                    self.O2, self.LSE2, scale=0.125, **kw)

    def outputs(self):
        return [self.O, self.LSE, self.O2, self.LSE2, self.index, self.length, self.count,
                self.table, *self.slot]


SESSIONS = [dict(seed=1), dict(seed=2, Lq=5, d=128, contract="strict_f32", page=32),
            dict(seed=3, B=2, Hq=12, H=1, n=3000, room=9000, d=128, page=64, keep=20),
            dict(seed=4, B=70, Hq=4, H=2, n=60, room=200, d=32, Lq=2),
            dict(seed=5, B=1, Hq=16, H=1, n=9000, room=20000, Lq=3, page=256, keep=9),
            dict(seed=8, B=300, Hq=4, H=2, n=700, room=1000, d=32)]


def expected(s):
    import torch
    s.reset()
    s.run()
    torch.cuda.synchronize()
    out = [t.clone() for t in s.outputs()]
    assert all(bool(torch.isfinite(t).all()) for t in (s.O, s.O2, s.LSE, s.LSE2))
    return out


def test_the_sessions_results(gpu_lib):
    """What the other tests compare with: tables, slots and attention of the first."""
    say("paged: session against the plain implementation")
    s = Session(gpu_lib, **SESSIONS[1])
    expected(s)
    host = lambda t: t.float().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()
    B, P = s.table.shape
    table, free = np.full((B, P), -1), host(s.start).copy()
    n, count = np.zeros(B, int), len(free)
    for k in range(2):
        n, count, slot, _ = ref.resize(n, host(s.want[k]), table, free, count, s.page, s.T[k])
        assert np.array_equal(host(s.slot[k]), slot)
    assert np.array_equal(host(s.table), table) and int(s.count) == count
    N, H, page, d = s.Kp.shape
    K = np.full((N, H, page, d), np.nan, np.float32)
    V, bounds = K.copy(), np.full((N, H, 2, d), np.nan, np.float32)
    for k in range(2):
        ref.append(*(host(x) for x in s.rows[k]), K, V, bounds, host(s.slot[k]), "f32")
    Q, O, LSE = host(s.Q), host(s.O), host(s.LSE)
    for b in range(B):
        for hq in range(Q.shape[1]):
            for i in range(Q.shape[2]):
                j = np.arange(ref.limit(n[b], Q.shape[2], i, True))
                at, row, h = table[b, j // page], j % page, hq // (Q.shape[1] // H)
                rO, rL, tO, tL = ref.attention(Q[b, hq, i], K[at, h, row], V[at, h, row], 0.125,
                                               "f32")
                assert abs(LSE[b, hq, i] - rL) <= tL and np.all(np.abs(O[b, hq, i] - rO) <= tO)


def test_sessions_captured_in_a_graph(gpu_lib):
    import torch
    say("paged: sessions captured and replayed")
    sessions = [Session(gpu_lib, **k) for k in SESSIONS]
    want = [expected(s) for s in sessions]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, capture_error_mode="relaxed"):
        for s in sessions:
            s.run()
    scratch = torch.randn(1 << 20, device="cuda")
    for rep in range(3):
        for s in sessions:
            s.reset()
        scratch.sin_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for k, (s, w) in enumerate(zip(sessions, want)):
            assert same(s.outputs(), w), (rep, k)


@pytest.mark.parametrize("B", [100, 300])
def test_captured_attention_follows_the_lengths_of_many_sequences(gpu_lib, B):
    """Units that every wave finds, and that a kernel writes down, are the replay's."""
    import torch
    mg = gpu_lib
    say("paged: captured attention of %d sequences" % B)
    rng = np.random.default_rng(22)
    Hq, H, d, page, P = 2, 1, 32, 16, 300
    N = B * P // 8
    Kp, Vp = (randn(rng, N, H, page, d) for _ in range(2))
    Q = randn(rng, B, Hq, 1, d)
    table = ints(*rng.integers(0, N, B * P)).view(B, P)
    length, O, LSE = ints(*[0] * B), torch.empty_like(Q), torch.empty(B, Hq, 1, device="cuda")
    ws = torch.empty(mg.mg_attn_fwd_paged_workspace_bytes(B, Hq, H, 1, d, page, P),
                     dtype=torch.uint8, device="cuda")
    call = lambda O, LSE, ws: mg.mg_attn_fwd_paged(Q, Kp, Vp, table, length, O, LSE, causal=True,
                                                   scale=0.2, workspace=ws)
    call(O, LSE, ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, capture_error_mode="relaxed"):
        call(O, LSE, ws)
    for most in (4800, 1, 900, 0, 4800):
        n = rng.integers(0, most + 1, B)
        n[rng.integers(B)] = most
        length.copy_(ints(*n))
        O.fill_(math.nan)
        LSE.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        got = [O.clone(), LSE.clone()]
        call(O, LSE, None)
        torch.cuda.synchronize()
        assert same(got, [O, LSE]), most
        assert bool((torch.isinf(LSE[:, 0, 0]) == (length == 0)).all())
        assert bool(torch.isfinite(O).all())


def test_a_captured_step_follows_the_lengths(gpu_lib):
    """One graph of a decode step, replayed while sequences grow over page borders:
    lengths, tables and grids are the device's."""
    import torch
    mg = gpu_lib
    say("paged: a captured step")
    rng = np.random.default_rng(21)
    B, Hq, H, d, page, P = 4, 8, 2, 64, 16, 500
    N = B * P
    Kp, Vp, bounds = mg.paged_cache(N, H, page, d)
    table, free = torch.zeros(B, P, dtype=torch.int32, device="cuda"), ints(*rng.permutation(N))
    length, count, want = ints(0, 0, 0, 0), ints(N), ints(0, 0, 0, 0)
    first = ints(13, 700, 0, 4100)
    T = int(first.sum())
    slot, offset = torch.empty(T, dtype=torch.int32, device="cuda"), ints(0, 0, 0, 0, 0)
    mg.mg_paged_resize(length, first, table, free, count, length, count, slot, offset, page=page)
    mg.mg_paged_append(randn(rng, T, H, d), randn(rng, T, H, d), Kp, Vp, slot, bounds)
    K, V, Q = randn(rng, B, H, d), randn(rng, B, H, d), randn(rng, B, Hq, 1, d)
    step, O = ints(0, 0, 0, 0), torch.empty_like(Q)
    LSE = torch.empty(B, Hq, 1, device="cuda")
    sizes = (B, Hq, H, 1, d, page, P)
    ws = torch.empty(mg.mg_attn_fwd_paged_workspace_bytes(*sizes), dtype=torch.uint8, device="cuda")

    def run():
        want.copy_(length)
        want.add_(1)
        mg.mg_paged_resize(length, want, table, free, count, length, count, step, offset, page=page)
        mg.mg_paged_append(K, V, Kp, Vp, step, bounds)
        mg.mg_attn_fwd_paged(Q, Kp, Vp, table, length, O, LSE, causal=True, scale=0.125, workspace=ws)

    graph = torch.cuda.CUDAGraph()
    state = [t.clone() for t in (length, table, free, count, Kp, Vp)]
    with torch.cuda.graph(graph, capture_error_mode="relaxed"):
        run()
    replayed = []
    for _ in range(40):
        K.mul_(-0.9)
        Q.add_(0.01)
        graph.replay()
        replayed.append((O.clone(), LSE.clone(), length.clone()))
    torch.cuda.synchronize()
    for t, old in zip((length, table, free, count, Kp, Vp), state):
        t.copy_(old)
    assert [int(x) for x in replayed[-1][2]] == [53, 740, 40, 4140]
    # K and Q went through the same roundings: run the eager steps on the same values
    rng = np.random.default_rng(21)
    rng.permutation(N)
    randn(rng, T, H, d), randn(rng, T, H, d)
    for t in (K, V, Q):
        t.copy_(randn(rng, *t.shape))
    for O1, LSE1, length1 in replayed:
        K.mul_(-0.9)
        Q.add_(0.01)
        run()
        assert torch.equal(O, O1) and torch.equal(LSE, LSE1) and torch.equal(length, length1)


def test_two_graphs_share_a_workspace(gpu_lib):
    """Replayed one after the other, in either order."""
    import torch
    say("paged: two graphs and one workspace")
    a, b = (Session(gpu_lib, **SESSIONS[k]) for k in (2, 4))
    ws = torch.empty(max(a.ws.numel(), b.ws.numel()), dtype=torch.uint8, device="cuda")
    a.ws = b.ws = ws
    want = [expected(s) for s in (a, b)]
    graphs = []
    for s in (a, b):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], capture_error_mode="relaxed"):
            s.run()
    for order in ((0, 1), (1, 0), (0, 1)):
        a.reset()
        b.reset()
        for k in order:
            graphs[k].replay()
        torch.cuda.synchronize()
        assert same(a.outputs(), want[0]) and same(b.outputs(), want[1]), order


@pytest.mark.parametrize("workspace", [True, False])
def test_sessions_on_streams(gpu_lib, workspace):
    import torch
    say("paged: sessions on streams, own workspace %s" % workspace)
    sessions = [Session(gpu_lib, **k) for k in SESSIONS]
    want = [expected(s) for s in sessions]
    streams = [torch.cuda.Stream() for _ in sessions]
    for rep in range(3):
        for s in sessions:
            s.reset()
        torch.cuda.synchronize()
        for s, st in zip(sessions, streams):
            s.run(st, workspace)
            torch.full((1 << 20,), float("nan"), device="cuda")   # memory the binding let go
        torch.cuda.synchronize()
        for k, (s, w) in enumerate(zip(sessions, want)):
            assert same(s.outputs(), w), (rep, k)


def test_a_device_that_is_not_the_current_one(gpu_lib):
    import torch
    if torch.cuda.device_count() < 2:
        pytest.skip("one GPU")
    a, b = (Session(gpu_lib, device="cuda:%d" % k, **SESSIONS[0]) for k in range(2))
    with torch.cuda.device(0):
        want = expected(a)
        b.reset()
        torch.cuda.synchronize(1)
        b.run()
        torch.cuda.synchronize(1)
    assert same([t.to("cuda:0") for t in b.outputs()], want)


@pytest.mark.parametrize("kwargs", SESSIONS + [
    dict(seed=6, B=1, Hq=1, H=1, n=15, room=16, d=32, keep=2),
    dict(seed=7, B=2, Hq=6, H=6, n=33, room=40, d=128, Lq=2, contract="strict_f32"),
    dict(seed=8, B=2, Hq=34, H=2, n=500, room=600, d=128, Lq=4, page=128)])
def test_nothing_outside_the_buffers_is_written(gpu_lib, kwargs):
    import torch
    say("paged: guards %s" % kwargs)
    s = Session(gpu_lib, **kwargs)
    want = expected(s)
    s.reset()
    wholes = []
    for name in ("Kp", "Vp", "bounds", "Q", "table", "free", "count", "length", "offset", "index", "O",
                 "O2", "LSE", "LSE2", "ws"):
        view, whole = guarded(getattr(s, name))
        setattr(s, name, view)
        wholes.append((name, whole))
    for k in range(2):
        s.slot[k], whole = guarded(s.slot[k])
        wholes.append(("slot", whole))
        s.rows[k] = [guarded(t)[0] for t in s.rows[k]]
    Q = s.Q.clone()
    s.run()
    torch.cuda.synchronize()
    assert same(s.outputs(), want) and torch.equal(s.Q, Q)
    for name, whole in wholes:
        assert bool((whole[:GUARD] == 0xA5).all()) and bool((whole[-GUARD:] == 0xA5).all()), name


@pytest.mark.parametrize("contract", ["fast_bf16", "strict_f32"])
def test_pools_beyond_32_bit_offsets(gpu_lib, contract):
    """Pools of 9.7 GB, pages from both ends: as in small pools with the same pages."""
    import torch
    mg = gpu_lib
    say("paged: 9.7 GB pools %s" % contract)
    rng = np.random.default_rng(9)
    elem = torch.bfloat16 if contract == "fast_bf16" else torch.float32
    B, Hq, H, d, page, P, n = 2, 8, 8, 128, 64, 40, 2500
    N = 74000 if contract == "fast_bf16" else 37000
    few = 2 * P
    big, small = mg.paged_cache(N, H, page, d, contract), mg.paged_cache(few, H, page, d, contract)
    assert big[0].numel() * big[0].element_size() > 9 << 30
    table = rng.permutation(few).reshape(B, P)
    far = np.where(table < P, table, N - few + table)
    length = ints(n, n - 700)
    pos = np.arange(n)
    K, V = randn(rng, 2 * n, H, d, dtype=elem), randn(rng, 2 * n, H, d, dtype=elem)
    Q = randn(rng, B, Hq, 1, d, dtype=elem)
    out = []
    for (Kp, Vp, bounds), t in ((big, far), (small, table)):
        slot = ints(*np.concatenate([t[b, pos // page] * page + pos % page for b in range(B)]))
        mg.mg_paged_append(K, V, Kp, Vp, slot, bounds, contract=contract)
        t = torch.tensor(t, dtype=torch.int32, device="cuda")
        kw = dict(causal=True, scale=0.1, contract=contract)
        out.append(mg.attention_forward_paged(Q, Kp, Vp, t, length, **kw) +
                   mg.attention_forward_paged(Q, Kp, Vp, t, length, bounds=bounds, keep=7, **kw))
        pages = t[0, :ref.pages(n, page)].long()
        out[-1] += (Kp[pages][:, :, :n % page], Vp[pages][:, :, :n % page], bounds[pages])
    assert same(*out)


def test_results_do_not_change_from_call_to_call(gpu_lib):
    import torch
    say("paged: the same bits again")
    for kwargs in SESSIONS:
        s = Session(gpu_lib, **kwargs)
        want = expected(s)
        for _ in range(3):
            s.reset()
            s.run()
            torch.cuda.synchronize()
            assert same(s.outputs(), want)


def test_a_million_tokens(gpu_lib):
    """One page, listed over and over, stands for 2^20 + 5 equal tokens: sums of terms
    that are all alike do not drift.  A wave adds at most 128 blocks of 8 values a lane
    (sparse: 64 pages a unit) and 512 units are joined: fewer than 2^11 roundings, each
    at most 2^-24, in the row's sum and in O's."""
    import torch
    mg = gpu_lib
    say("paged: a million tokens")
    n, page, d = (1 << 20) + 5, 256, 32
    P, drift = ref.pages(n, page), 2.0 ** -13
    for contract, elem, step in (("fast_bf16", torch.bfloat16, 2.0 ** -8),
                                 ("strict_f32", torch.float32, 2.0 ** -24)):
        Kp, Vp = (torch.full((1, 1, page, d), x, dtype=elem, device="cuda") for x in (0.5, 0.7))
        table = torch.zeros(1, P, dtype=torch.int32, device="cuda")
        Q = torch.full((1, 2, 1, d), 0.25, dtype=elem, device="cuda")
        every = torch.arange(P, dtype=torch.int32, device="cuda").view(1, 1, 1, P)
        for index in (None, every):
            O, LSE = torch.empty_like(Q), torch.empty(1, 2, 1, device="cuda")
            kw = dict(causal=True, scale=1.0, contract=contract)
            if index is None:
                mg.mg_attn_fwd_paged(Q, Kp, Vp, table, ints(n), O, LSE, **kw)
            else:
                mg.mg_attn_fwd_paged_sparse(Q, Kp, Vp, table, ints(n), index, O, LSE, **kw)
            assert float((O.double() / Vp[0, 0, 0].double() - 1).abs().max()) <= step + 2 * drift
            # a score is 4 exactly; LSE is below 18, and rounded a few times
            assert float((LSE.double() - 4 - math.log(n)).abs().max()) <= drift + 18 * 2.0 ** -22


def test_many_sequences(gpu_lib):
    """40,000 sequences of none to 90 tokens, of which every one is as it is alone."""
    import torch
    mg = gpu_lib
    say("paged: 40,000 sequences")
    rng = np.random.default_rng(17)
    B, Hq, H, d, page, P, N = 40000, 2, 1, 32, 16, 6, 500
    Kp, Vp, Q = randn(rng, N, H, page, d), randn(rng, N, H, page, d), randn(rng, B, Hq, 1, d)
    table = torch.from_numpy(rng.integers(0, N, (B, P)).astype(np.int32)).cuda()
    length = torch.from_numpy(rng.integers(0, 91, B).astype(np.int32)).cuda()
    O, LSE = mg.attention_forward_paged(Q, Kp, Vp, table, length, causal=True, scale=0.2)
    k, v = (x.float()[table.long(), 0].reshape(B, P * page, d) for x in (Kp, Vp))
    S = (Q[:, :, 0].double() @ k.double().transpose(1, 2).contiguous()) * 0.2
    S.masked_fill_(torch.arange(P * page, device="cuda") >= length[:, None, None], -math.inf)
    z = torch.logsumexp(S, 2)
    want = torch.exp(S - torch.where(z.isneginf(), 0.0, z)[..., None]) @ v.double()
    assert torch.equal(z.isneginf(), LSE[:, :, 0].isneginf())
    fin = ~z.isneginf()
    assert float((LSE[:, :, 0].double() - z)[fin].abs().max()) <= 1e-5
    # 2^-8 of the value for bf16, 1e-4 for all else (|v| below 6, scores off by 1e-6)
    off = (O[:, :, 0].double() - want).abs() - 2.0 ** -8 * want.abs()
    assert float(off.max()) <= 1e-4


def test_refusals(gpu_lib):
    import torch
    mg = gpu_lib
    say("paged: refusals")
    rng = np.random.default_rng(10)
    B, Hq, H, page, d, P, N, T = 2, 4, 2, 16, 64, 5, 12, 6
    Kp, Vp, bounds = mg.paged_cache(N, H, page, d)
    K, Q, LSE = randn(rng, T, H, d), randn(rng, B, Hq, 1, d), torch.empty(B, Hq, 1, device="cuda")
    O = torch.empty_like(Q)
    slot, table, length = ints(*range(T)), torch.zeros(B, P, device="cuda").int(), ints(5, 3)
    free, one, off = ints(*range(N)), ints(N), ints(0, 0, 0)
    index = torch.zeros(B, H, 1, 4, device="cuda").int()
    kw = dict(causal=True, scale=1.0)
    sel = dict(page=page, causal=True, first=1, recent=1)

    def resize(key_len=length, want=length, table=table, free=free, count=one, new_len=length,
               new_count=one, slot=slot, offset=off, **k):
        mg.mg_paged_resize(key_len, want, table, free, count, new_len, new_count, slot, offset,
                           **{"page": page, **k})

    wrong = [
        (lambda: resize(want=length.long()), "dtype"), (lambda: resize(want=ints(1)), "shape"),
        (lambda: resize(offset=ints(0, 0)), "shape"), (lambda: resize(count=ints(1, 2)), "shape"),
        (lambda: resize(table=table.T), "contiguous"), (lambda: resize(table=table.cpu()), "GPU"),
        (lambda: resize(slot=slot[::2]), "contiguous"), (lambda: resize(free=free.cpu()), "GPU"),
        (lambda: mg.mg_paged_append(K, K.float(), Kp, Vp, slot), "dtype"),
        (lambda: mg.mg_paged_append(K, K, Kp, Vp, slot, contract="strict_f32"), "dtype"),
        (lambda: mg.mg_paged_append(K, K[:4], Kp, Vp, slot), "shape"),
        (lambda: mg.mg_paged_append(K, K, Kp, Vp[:4], slot), "shape"),
        (lambda: mg.mg_paged_append(K, K, Kp, Vp, slot[:5]), "shape"),
        (lambda: mg.mg_paged_append(K, K, Kp, Vp, slot, bounds[:5]), "shape"),
        (lambda: mg.mg_paged_append(K, K, Kp.transpose(2, 3), Vp, slot), "rows are"),
        (lambda: mg.mg_paged_append(K.transpose(0, 1).contiguous().transpose(0, 1), K, Kp, Vp, slot),
         "contiguous"),
        (lambda: mg.mg_attn_fwd_paged(Q, Kp, Vp, table, length, O, LSE[..., 0], **kw), "shape"),
        (lambda: mg.mg_attn_fwd_paged(Q, Kp, Vp, table[:1], length, O, LSE, **kw), "sequences"),
        (lambda: mg.mg_attn_fwd_paged(Q, Kp, Vp, table[:, ::2], length, O, LSE, **kw), "contiguous"),
        (lambda: mg.mg_attn_fwd_paged(Q, Kp, Vp, table, length, O, LSE, ints(1), **kw), "shape"),
        (lambda: mg.mg_attn_fwd_paged(Q, Kp, Vp, table, length, O, LSE, **kw,
                                      workspace=torch.empty(8)), "workspace"),
        (lambda: mg.mg_attn_fwd_paged_sparse(Q, Kp, Vp, table, length, index[:, :1], O, LSE, **kw),
         "shape"),
        (lambda: mg.mg_paged_select(Q, bounds[:, :, :1], table, length, index, **sel), "shape"),
        (lambda: mg.mg_paged_select(Q, bounds.float(), table, length, index, **sel), "dtype"),
        (lambda: mg.mg_paged_select(Q, bounds, table, length, index[:1], **sel), "shape"),
    ]
    for call, word in wrong:
        with pytest.raises(ValueError, match=word):
            call()
    bad = [
        (lambda: resize(page=20), 2),
        (lambda: mg.mg_attn_fwd_paged(Q[:, :3].contiguous(), Kp, Vp, table, length,
                                      O[:, :3].contiguous(), LSE[:, :3].contiguous(), **kw), 1),
        (lambda: mg.mg_attn_fwd_paged(Q, Kp, Vp, table, length, O, LSE, causal=True,
                                      scale=math.inf), 1),
        (lambda: mg.mg_paged_select(Q, bounds, table, length, index, page=page, causal=True, first=3,
                                    recent=2), 1),
        (lambda: mg.mg_paged_select(Q, bounds, table, length, index, **sel,
                                    workspace=torch.empty(16, dtype=torch.uint8, device="cuda")), 4),
        (lambda: mg.mg_paged_append(randn(rng, T, H, 16), randn(rng, T, H, 16),
                                    *(randn(rng, N, H, page, 16) for _ in range(2)), slot), 2),
    ]
    for call, status in bad:
        with pytest.raises(mg.MgError) as e:
            call()
        assert e.value.status == status
