"""How a program uses the 4-bit cache: inside guarded buffers, captured into a
graph, on several streams, with lengths that need clamping, beyond 4 GiB; and
what its entry points refuse."""
import math

import numpy as np
import pytest

import kv4_ref as ref
from gpu_util import say

pytestmark = pytest.mark.gpu


def bf16(rng, *shape):
    import torch
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).cuda().bfloat16()


def ints(*x):
    import torch
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Session:
    """One sequence batch and its buffers: tokens in, attention with weights,
    eviction in place."""

    def __init__(self, mg, seed, B=2, Hq=8, H=2, L=700, d=64, n=500, Lq=3, keep=300,
                 contract="fast_bf16"):
        import torch
        rng = np.random.default_rng(seed)
        self.mg, self.d, self.L, self.H, self.n, self.contract = mg, d, L, H, n, contract
        elem = torch.bfloat16 if contract == "fast_bf16" else torch.float32
        self.K, self.V, self.Q = (bf16(rng, B, h, m, d).to(elem)
                                  for h, m in ((H, n), (H, n), (Hq, Lq)))
        self.cache = mg.kv4_cache(B, H, L, d)
        self.weight = torch.empty(B, H, L, device="cuda")
        self.length = ints(*([n] * B))
        self.index = torch.empty(B, H, keep, dtype=torch.int32, device="cuda")
        self.O, self.LSE = torch.empty_like(self.Q), torch.empty(B, Hq, Lq, device="cuda")
        need = mg.mg_attn_fwd_kv4_workspace_bytes(B, Hq, H, Lq, L, d, True, contract)
        self.ws = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
        self.outK, self.outV = (torch.zeros(B, H, n, d, dtype=elem, device="cuda")
                                for _ in range(2))

    def reset(self):
        self.cache.zero_()
        self.weight.fill_(float("nan"))
        self.length.fill_(self.n)
        for t in (self.O, self.LSE, self.outK, self.outV):
            t.zero_()

    def run(self, stream=None, workspace=True):
        mg, kw = self.mg, dict(contract=self.contract, stream=stream)
        mg.mg_kv4_append(self.K, self.V, self.cache, L=self.L, weight=self.weight, **kw)
        mg.mg_attn_fwd_kv4(self.Q, self.cache, self.O, self.LSE, self.length, H=self.H, L=self.L,
                           causal=True, scale=0.125, weight=self.weight,
                           workspace=self.ws if workspace else None, **kw)
        mg.mg_kv4_evict(self.cache, self.weight, self.index, self.length, self.length, d=self.d,
                        recent=min(20, self.index.shape[2]), stream=stream)
        mg.mg_kv4_read(self.cache, self.outK, self.outV, None, self.length, L=self.L, **kw)

    def outputs(self):
        n = self.index.shape[2]
        return [self.O, self.LSE, self.index, self.length, self.weight[:, :, :n], self.outK,
                self.outV]


# few rows with kept scores; rows whose weights are recomputed; many rows
SESSIONS = [dict(seed=1), dict(seed=2, Lq=5, d=128, contract="strict_f32"),
            dict(seed=3, Lq=90, d=128), dict(seed=4, L=5000, n=4500, Lq=1, keep=900, d=32),
            dict(seed=8, B=1, Hq=16, H=4, L=9000, n=8500, Lq=241, keep=5000, d=128)]


def expected(s):
    import torch
    s.reset()
    s.run()
    torch.cuda.synchronize()
    return [t.clone() for t in s.outputs()]


def same(got, want):
    import torch
    return all(torch.equal(a, b) for a, b in zip(got, want))


def test_sessions_captured_in_a_graph(gpu_lib):
    import torch
    say("kv4: sessions captured and replayed")
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


@pytest.mark.parametrize("workspace", [True, False])
def test_sessions_on_streams(gpu_lib, workspace):
    import torch
    say("kv4: sessions on streams, own workspace %s" % workspace)
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


GUARD = 4096


def guarded(t):
    """A copy of t between guard bytes: (view, whole, fill)."""
    import torch
    raw = t.contiguous().view(torch.uint8).flatten() if t.dtype != torch.uint8 else t.flatten()
    whole = torch.full((raw.numel() + 2 * GUARD,), 0xA5, dtype=torch.uint8, device="cuda")
    whole[GUARD:GUARD + raw.numel()] = raw
    return whole[GUARD:GUARD + raw.numel()].view(t.dtype).view(t.shape), whole


@pytest.mark.parametrize("kwargs", SESSIONS + [
    dict(seed=5, B=1, Hq=1, H=1, L=33, n=33, Lq=1, keep=9, d=32),
    dict(seed=6, B=3, Hq=6, H=6, L=301, n=37, Lq=37, keep=21, d=64, contract="strict_f32"),
    dict(seed=7, B=1, Hq=4, H=1, L=129, n=129, Lq=129, keep=120, d=128)])
def test_nothing_outside_the_buffers_is_written(gpu_lib, kwargs):
    import torch
    say("kv4: guards %s" % kwargs)
    s = Session(gpu_lib, **kwargs)
    want = expected(s)
    s.reset()
    wholes = []
    for name in ("K", "V", "Q", "cache", "weight", "length", "index", "O", "LSE", "ws", "outK",
                 "outV"):
        view, whole = guarded(getattr(s, name))
        setattr(s, name, view)
        wholes.append((name, whole))
    inputs = [t.clone() for t in (s.K, s.V, s.Q)]
    s.run()
    torch.cuda.synchronize()
    assert same(s.outputs(), want)
    assert same((s.K, s.V, s.Q), inputs)
    for name, whole in wholes:
        assert bool((whole[:GUARD] == 0xA5).all()) and bool((whole[-GUARD:] == 0xA5).all()), name


@pytest.mark.parametrize("Lq,L", [(1, 90), (40, 90), (1400, 6100)])
def test_lengths_are_clamped(gpu_lib, Lq, L):
    """Lengths above what there is, and below 0, mean all of it and nothing."""
    import torch
    mg = gpu_lib
    say("kv4: lengths out of range, Lq%d" % Lq)
    rng = np.random.default_rng(8)
    B, Hq, H, d = 3, 4, 2, 64
    cache = mg.kv4_cache(B, H, L, d)
    K, V = bf16(rng, B, H, L, d), bf16(rng, B, H, L, d)
    mg.mg_kv4_append(K, V, cache, None, ints(1 << 30, L, L), L=L)
    Q = bf16(rng, B, Hq, Lq, d)

    def run(key_len, q_len):
        w = torch.zeros(B, H, L, device="cuda")
        O, LSE = mg.attention_forward_kv4(Q, cache, H=H, L=L, causal=True, scale=0.1,
                                          key_len=key_len, q_len=q_len, weight=w)
        return O, LSE, w

    a = run(ints(1 << 30, -7, 50), ints(Lq + 9, Lq, -3))
    b = run(ints(L, 0, 50), ints(Lq, Lq, 0))
    assert same(a, b)
    assert bool((a[0][1:] == 0).all()) and bool(torch.isneginf(a[1][1:]).all())
    assert bool((a[2][1:] == 0).all()) and bool(torch.isfinite(a[1][0]).all())


def test_a_cache_beyond_32_bit_offsets(gpu_lib):
    """A cache of 9.8 GB: the last head's tokens, written, read, attended and
    evicted, are those of a small cache with the same contents."""
    import torch
    mg = gpu_lib
    say("kv4: 9.8 GB cache")
    rng = np.random.default_rng(9)
    H, L, d, keep = 520, 131072, 128, 1000
    n = 3000                                   # tokens written at the far end of every head
    K, V = (bf16(rng, 1, 1, n, d) for _ in range(2))
    big, small = mg.kv4_cache(1, H, L, d), mg.kv4_cache(1, 1, L, d)
    big.zero_()
    small.zero_()
    all_K, all_V = (t.expand(1, H, n, d).contiguous() for t in (K, V))
    mg.mg_kv4_append(all_K, all_V, big, ints(L - n), L=L)
    mg.mg_kv4_append(K, V, small, ints(L - n), L=L)
    outs = [torch.zeros_like(t) for t in (all_K, all_V, K, V)]
    mg.mg_kv4_read(big, outs[0], outs[1], ints(L - n), L=L)
    mg.mg_kv4_read(small, outs[2], outs[3], ints(L - n), L=L)
    for b, s in ((outs[0], outs[2]), (outs[1], outs[3])):
        assert torch.equal(b, s.expand_as(b))
    for Lq in (1, 64, 128):
        q = bf16(rng, 1, 1, Lq, d)
        wb, ws = torch.zeros(1, H, L, device="cuda"), torch.zeros(1, 1, L, device="cuda")
        kw = dict(L=L, causal=True, scale=0.2)
        Ob, Lb = mg.attention_forward_kv4(q.expand(1, H, Lq, d).contiguous(), big, H=H, weight=wb,
                                          **kw)
        Os, Ls = mg.attention_forward_kv4(q, small, H=1, weight=ws, **kw)
        # (the heads' tokens are split otherwise, so sums may differ in order)
        assert float((Ob.float() - Os.float()).abs().max()) <= 2.0 ** -7 * float(Os.abs().max())
        assert float((Lb - Ls).abs().max()) <= 1e-5 * float(Ls.abs().max())
        assert float((wb - ws).abs().max()) <= 1e-5 * float(ws.abs().max())
        assert torch.equal(Ob[0, 0], Ob[0, H - 1]) and torch.equal(wb[0, 0], wb[0, H - 1])
    index = torch.empty(1, H, keep, dtype=torch.int32, device="cuda")
    new = ints(0)
    mg.mg_kv4_evict(big, wb, index, new, d=d, recent=10)
    assert bool((index == index[:, :1]).all()) and int(new[0]) == keep
    at = index[0, 0].long() - (L - n)
    row = torch.zeros(1, H, keep, d, dtype=torch.bfloat16, device="cuda")
    row2 = torch.zeros_like(row)
    mg.mg_kv4_read(big, row, row2, L=L)
    assert torch.equal(row[0, H - 1], torch.where((at >= 0)[:, None],
                                                  outs[2][0, 0][at.clamp(min=0)], 0.0))


def test_the_most_heads(gpu_lib):
    """2^19 heads, whose grids come near 2^32 threads: every one as a single one."""
    import torch
    mg = gpu_lib
    say("kv4: 2^19 heads")
    rng = np.random.default_rng(13)
    B, H, L, d, n, keep = 1 << 10, 1 << 9, 32, 128, 21, 7

    def session(b, h, K, V, Q):
        cache, w = mg.kv4_cache(b, h, L, d), torch.zeros(b, h, L, device="cuda")
        k, v, q = (t.expand(b, h, -1, d).contiguous() for t in (K, V, Q))
        length = ints(*([n] * b))
        mg.mg_kv4_append(k, v, cache, L=L, weight=w)
        O, LSE = mg.attention_forward_kv4(q, cache, H=h, L=L, causal=True, scale=0.1,
                                          key_len=length, weight=w)
        index = torch.empty(b, h, keep, dtype=torch.int32, device="cuda")
        mg.mg_kv4_evict(cache, w, index, length, length, d=d, recent=2)
        out = torch.zeros(b, h, keep, d, dtype=torch.bfloat16, device="cuda")
        mg.mg_kv4_read(cache, out, torch.empty_like(out), L=L)
        return O, LSE, w[:, :, :n], index, out, length

    data = [bf16(rng, 1, 1, m, d) for m in (n, n, 1)]
    few, many = session(1, 1, *data), session(B, H, *data)
    for a, b in zip(few, many):
        assert bool((b == a).all())


def test_refusals(gpu_lib):
    import torch
    mg = gpu_lib
    say("kv4: refusals")
    rng = np.random.default_rng(10)
    B, H, n, L, d = 2, 2, 4, 40, 64
    K = bf16(rng, B, H, n, d)
    cache = mg.kv4_cache(B, H, L, d)
    Q, LSE = bf16(rng, B, 4, 1, d), torch.empty(B, 4, 1, device="cuda")
    w = torch.zeros(B, H, L, device="cuda")
    kw = dict(H=H, L=L, causal=True, scale=1.0)
    wrong = [
        (lambda: mg.mg_kv4_append(K, K, cache[:-256], L=L), "bytes"),
        (lambda: mg.mg_kv4_append(K, K.float(), cache, L=L), "dtype"),
        (lambda: mg.mg_kv4_append(K, K, cache, L=L, contract="strict_f32"), "dtype"),
        (lambda: mg.mg_kv4_append(K.transpose(1, 2), K.transpose(1, 2), cache, L=L), "contiguous"),
        (lambda: mg.mg_kv4_append(K, K[:, :, :2], cache, L=L), "shape"),
        (lambda: mg.mg_kv4_append(K, K, cache, ints(1), L=L), "shape"),
        (lambda: mg.mg_kv4_append(K, K, cache, ints(1, 2).long(), L=L), "dtype"),
        (lambda: mg.mg_kv4_append(K, K, cache.cpu(), L=L), "GPU"),
        (lambda: mg.mg_kv4_append(K, K, cache, L=L, weight=w[:, :, :5].contiguous()), "shape"),
        (lambda: mg.mg_kv4_append(K[0], K[0], cache, L=L), "B,H,n,d"),
        (lambda: mg.mg_attn_fwd_kv4(Q, cache, Q, LSE[..., 0], **kw), "shape"),
        (lambda: mg.mg_attn_fwd_kv4(Q[..., :32], cache, Q, LSE, **kw), "contiguous"),
        (lambda: mg.mg_attn_fwd_kv4(Q, cache, Q.clone(), LSE, **kw, workspace=torch.empty(8)),
         "workspace"),
        (lambda: mg.mg_kv4_evict(cache, w[0], ints(1), ints(1, 1), d=d, recent=0), "weight"),
        (lambda: mg.mg_kv4_evict(cache, w, torch.empty(B, H, 5, device="cuda"), ints(1, 1), d=d,
                                 recent=0), "dtype"),
        (lambda: mg.mg_kv4_evict(cache, w, torch.empty(B, H, 5, device="cuda").int(), ints(1, 1),
                                 d=d, recent=0, out_weight=w), "together"),
    ]
    for call, word in wrong:
        with pytest.raises(ValueError, match=word):
            call()
    bad = [
        (lambda: mg.mg_attn_fwd_kv4(Q[:, :3].contiguous(), cache, Q[:, :3].contiguous(),
                                    LSE[:, :3].contiguous(), **kw), 1),     # 3 heads over 2
        (lambda: mg.mg_attn_fwd_kv4(Q, cache, Q.clone(), LSE, H=H, L=L, causal=True,
                                    scale=math.inf), 1),
        (lambda: mg.mg_attn_fwd_kv4(Q, cache, Q.clone(), LSE, **kw, weight=w,
                                    workspace=torch.empty(16, dtype=torch.uint8, device="cuda")), 4),
        (lambda: mg.mg_kv4_evict(cache, w, torch.empty(B, H, 5, device="cuda").int(), ints(1, 1),
                                 d=d, recent=6), 1),
        (lambda: mg.mg_kv4_evict(cache, w, torch.empty(B, H, L + 1, device="cuda").int(),
                                 ints(1, 1), d=d, recent=6), 1),
    ]
    for call, status in bad:
        with pytest.raises(mg.MgError) as e:
            call()
        assert e.value.status == status
    # a cache may start at any 16-byte boundary
    whole = torch.zeros(cache.numel() + 64, dtype=torch.uint8, device="cuda")
    mg.mg_kv4_append(K, K, whole[16:16 + cache.numel()], L=L)
    mg.mg_kv4_append(K, K, cache, L=L)
    a, b = (mg.attention_forward_kv4(Q, c, key_len=ints(4, 3), **kw)
            for c in (whole[16:16 + cache.numel()], cache))
    assert same(a, b)
    with pytest.raises(mg.MgError) as e:
        mg.mg_kv4_append(K, K, whole[8:8 + cache.numel()], L=L)
    assert e.value.status == 3
