"""Host-side checks of the paged cache (no GPU needed): exported symbols, sizes,
refusals before anything is enqueued, the binding's own checks, and the tests'
plain implementation against the definition."""
import ctypes
import os
import re
import subprocess

import numpy as np
import pytest

import paged_ref as ref
import paper_2608_01563_amd as mg

vp = ctypes.c_void_p
GOOD = [0x1000 * (k + 1) for k in range(12)]   # aligned, never dereferenced


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(mg.LIB_PATH):
        pytest.fail("libmg.so is not built; run __graft_entry__.build()")
    return mg.load_library()


def test_every_declared_symbol_is_exported(lib):
    with open(mg.PAGED_HEADER_PATH) as f:
        text = re.sub(r"/\*.*?\*/", "", f.read(), flags=re.S)
    names = set(re.findall(r"\b(mg_[a-z0-9_]+)\s*\(", text))
    assert {"mg_paged_resize", "mg_paged_resize_workspace_bytes", "mg_paged_append",
            "mg_attn_fwd_paged", "mg_attn_fwd_paged_workspace_bytes", "mg_paged_select",
            "mg_paged_select_workspace_bytes", "mg_attn_fwd_paged_sparse",
            "mg_attn_fwd_paged_sparse_workspace_bytes"} == names
    out = subprocess.run(["nm", "-D", "--defined-only", mg.LIB_PATH], capture_output=True,
                         text=True, check=True).stdout
    exported = {line.split()[-1] for line in out.splitlines() if " T " in line}
    assert names <= exported
    assert all(hasattr(mg, n) for n in names)


def resize(lib, ptrs=GOOD, B=2, page=16, P=4, N=9, T=40, ws=0x9000, nbytes=1 << 20):
    return lib.mg_paged_resize(*(vp(p) for p in ptrs[:9]), B, page, P, N, T, vp(ws), nbytes, None)


def append(lib, ptrs=GOOD, T=3, H=2, d=64, page=16, N=9, contract=1):
    return lib.mg_paged_append(*(vp(p) for p in ptrs[:6]), T, H, d, page, N, contract, None)


def attn(lib, ptrs=GOOD, B=1, Hq=4, H=2, Lq=1, d=64, page=16, P=4, N=9, scale=0.125, contract=1,
         ws=0x9000, nbytes=1 << 30):
    return lib.mg_attn_fwd_paged(*(vp(p) for p in ptrs[:8]), B, Hq, H, Lq, d, page, P, N, 1,
                                 ctypes.c_float(scale), contract, vp(ws), nbytes, None)


def sparse(lib, ptrs=GOOD, B=1, Hq=4, H=2, Lq=1, d=64, page=16, P=4, N=9, keep=4, scale=0.125,
           contract=1, ws=0x9000, nbytes=1 << 30):
    return lib.mg_attn_fwd_paged_sparse(*(vp(p) for p in ptrs[:9]), B, Hq, H, Lq, d, page, P, N, 1,
                                        keep, ctypes.c_float(scale), contract, vp(ws), nbytes,
                                        None)


def select(lib, ptrs=GOOD, B=1, Hq=4, H=2, Lq=1, d=64, page=16, P=4, N=9, keep=4, first=1,
           recent=2, contract=1, ws=0x9000, nbytes=1 << 30):
    return lib.mg_paged_select(*(vp(p) for p in ptrs[:6]), B, Hq, H, Lq, d, page, P, N, 1, keep,
                               first, recent, contract, vp(ws), nbytes, None)


@pytest.mark.parametrize("call", [resize, append, attn, sparse, select])
def test_good_sizes_are_refused_for_their_pointers_only(lib, call):
    assert call(lib) == 1 and "device" in mg.mg_last_error_detail()


@pytest.mark.parametrize("kwargs,status", [
    (dict(B=0), 1), (dict(P=0), 1), (dict(N=0), 1), (dict(T=0), 1), (dict(page=24), 2),
    (dict(page=8), 2), (dict(page=512), 2), (dict(page=-16), 2), (dict(B=(1 << 16) + 1), 1),
    (dict(P=(1 << 20) + 1), 1), (dict(B=1 << 16, P=1 << 16), 1), (dict(N=1 << 27), 1),
    (dict(T=(1 << 28) + 1), 1), (dict(T=1 << 20, ws=0), 4), (dict(T=1 << 20, nbytes=8), 4),
    (dict(B=2000, nbytes=0), 4)])
def test_resize_refuses_bad_sizes(lib, kwargs, status):
    assert resize(lib, **kwargs) == status
    assert mg.mg_last_error_detail() != ""


@pytest.mark.parametrize("kwargs,status", [
    (dict(T=0), 1), (dict(H=0), 1), (dict(N=-1), 1), (dict(d=96), 2), (dict(d=0), 1),
    (dict(page=0), 2), (dict(contract=3), 1), (dict(contract=-1), 1), (dict(T=(1 << 27) + 1), 1),
    (dict(N=1 << 27), 1), (dict(H=1 << 14, page=256), 1)])
def test_append_refuses_bad_sizes(lib, kwargs, status):
    assert append(lib, **kwargs) == status
    assert mg.mg_last_error_detail() != ""


ROWS = [
    (dict(B=0), 1), (dict(Hq=0), 1), (dict(Hq=3), 1), (dict(Hq=1), 1), (dict(H=0), 1),
    (dict(Lq=0), 1), (dict(P=0), 1), (dict(N=0), 1), (dict(d=16), 2), (dict(page=48), 2),
    (dict(contract=7), 1), (dict(B=1 << 10, Hq=1 << 10, H=1 << 4, Lq=1 << 10), 1),
    (dict(B=1 << 10, Hq=1 << 10, H=1 << 10), 1), (dict(P=1 << 21), 1),
    (dict(B=1 << 16, P=1 << 16), 1)]


@pytest.mark.parametrize("call", [attn, sparse, select])
@pytest.mark.parametrize("kwargs,status", ROWS)
def test_queries_refuse_bad_sizes(lib, call, kwargs, status):
    assert call(lib, **kwargs) == status
    assert mg.mg_last_error_detail() != ""


@pytest.mark.parametrize("call,kwargs,status", [
    (attn, dict(scale=float("inf")), 1), (attn, dict(scale=float("nan")), 1),
    (attn, dict(scale=3e38), 1), (attn, dict(P=1 << 12, ws=0), 4),
    (attn, dict(P=1 << 12, nbytes=64), 4), (attn, dict(B=1 << 14, H=32, Hq=32, P=1 << 16), 1),
    (attn, dict(B=1 << 10, H=1 << 9, Hq=1 << 16, d=32, P=1 << 9), 1),   # rows to join
    (sparse, dict(B=1 << 10, H=1 << 9, Hq=1 << 16, d=32, keep=512), 1),
    (sparse, dict(keep=0), 1), (sparse, dict(keep=1 << 21), 1),
    (sparse, dict(scale=float("nan")), 1), (sparse, dict(keep=999, ws=0), 4),
    (select, dict(keep=0), 1), (select, dict(first=-1), 1), (select, dict(recent=-1), 1),
    (select, dict(first=3, recent=2), 1), (select, dict(first=2 ** 31 - 1, recent=1), 1),
    (select, dict(nbytes=16), 4), (select, dict(ws=0), 4),
    (select, dict(B=1 << 12, H=128, Hq=128, P=2048), 1)])
def test_queries_refuse_bad_arguments(lib, call, kwargs, status):
    assert call(lib, **kwargs) == status
    assert mg.mg_last_error_detail() != ""


def test_lists_that_a_row_could_not_count_are_refused(lib):
    # (a workgroup's threads go on from keep - 1 by up to 1,024)
    assert select(lib, Hq=1, H=1, keep=(1 << 31) - 1) == 1
    assert "too many scores" in mg.mg_last_error_detail()
    assert select(lib, Hq=1, H=1, keep=1 << 29) == 1   # in range: only the pointers are none
    assert "too many scores" not in mg.mg_last_error_detail()


@pytest.mark.parametrize("call,wide,narrow,optional", [
    (resize, (), range(9), ()), (append, (0, 1, 2, 3), (5,), (4,)),
    (attn, range(5), (5, 6), (7,)), (sparse, range(5), (5, 6, 7), (8,)),
    (select, (0, 1), (2, 3, 5), (4,))])
def test_bad_pointers_are_refused(lib, call, wide, narrow, optional):
    for k in (*wide, *narrow):
        ptrs = list(GOOD)
        ptrs[k] = 0
        assert call(lib, ptrs) == 1 and "NULL" in mg.mg_last_error_detail()
    for k, off in [(k, 8) for k in wide] + [(k, 2) for k in narrow]:
        ptrs = list(GOOD)
        ptrs[k] += off
        assert call(lib, ptrs) == 3
    bufs = [ctypes.create_string_buffer(4096) for _ in range(9)]
    host = [(ctypes.addressof(b) + 15) // 16 * 16 for b in bufs]
    for k in optional:
        host[k] = 0
    assert call(lib, host) == 1 and "device" in mg.mg_last_error_detail()


def test_workspace_queries():
    f = mg.mg_attn_fwd_paged_workspace_bytes
    assert f(1, 4, 4, 1, 64, 16, 16) == 0                  # one unit a sequence
    assert f(1, 8, 1, 1, 128, 64, 1 << 10) > 0
    assert f(64, 32, 8, 1, 128, 16, 1 << 10) > 0
    assert mg.mg_attn_fwd_paged_sparse_workspace_bytes(2048, 32, 8, 1, 128, 64, 8) == 0
    assert mg.mg_attn_fwd_paged_sparse_workspace_bytes(1, 8, 1, 1, 128, 64, 64) > 0
    assert mg.mg_paged_select_workspace_bytes(2, 8, 2, 3, 128, 64, 100) == -(-2 * 2 * 3 * 400 //
                                                                            256) * 256
    for bad in ((1, 5, 4, 1, 64, 16, 4), (1, 4, 4, 0, 64, 16, 4), (1, 4, 4, 1, 96, 16, 4),
                (1, 4, 4, 1, 64, 20, 4), (0, 4, 4, 1, 64, 16, 4), (1, 4, 0, 1, 64, 16, 4)):
        assert f(*bad) == mg.mg_paged_select_workspace_bytes(*bad) == 0
        assert mg.mg_attn_fwd_paged_sparse_workspace_bytes(*bad) == 0
    assert f(1, 8, 1, 1, 128, 64, 1 << 10, contract=9) == 0
    r = mg.mg_paged_resize_workspace_bytes
    assert r(4, 100) == 0 and r(4, 1 << 20) > 0 and r(1 << 15, 8) >= 5 * 4 << 15
    for B, T in ((0, 1), (1, 0), (-1, 5), ((1 << 16) + 1, 1), (1, (1 << 28) + 1)):
        assert r(B, T) == 0


def test_binding_refuses_what_is_not_on_the_gpu(lib):
    import torch
    i = torch.zeros(2, dtype=torch.int32)
    one = torch.zeros(1, dtype=torch.int32)
    table = torch.zeros(2, 3, dtype=torch.int32)
    Kp, Vp, bounds = mg.paged_cache(5, 2, 16, 64, device="cpu")
    assert Kp.shape == Vp.shape == (5, 2, 16, 64) and bounds.shape == (5, 2, 2, 64)
    assert mg.paged_cache(5, 2, 16, 64, "strict_f32", bounds=False, device="cpu")[2] is None
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    q = torch.zeros(2, 4, 1, 64, dtype=torch.bfloat16)
    index = torch.zeros(2, 2, 1, 2, dtype=torch.int32)
    lse = torch.zeros(2, 4, 1)
    with pytest.raises(ValueError, match="GPU"):
        mg.mg_paged_resize(i, i, table, i, one, i, one, i, i, page=16)
    with pytest.raises(ValueError, match="GPU"):
        mg.mg_paged_append(x, x, Kp, Vp, i)
    with pytest.raises(ValueError, match="GPU"):
        mg.mg_attn_fwd_paged(q, Kp, Vp, table, i, q, lse, causal=True, scale=1.0)
    with pytest.raises(ValueError, match="GPU"):
        mg.mg_attn_fwd_paged_sparse(q, Kp, Vp, table, i, index, q, lse, causal=True, scale=1.0)
    with pytest.raises(ValueError, match="GPU"):
        mg.mg_paged_select(q, bounds, table, i, index, page=16, causal=True, first=0, recent=0)


def test_binding_refuses_bad_shapes(lib):
    import torch
    i = torch.zeros(2, dtype=torch.int32)
    table = torch.zeros(2, 3, dtype=torch.int32)
    Kp, Vp, bounds = mg.paged_cache(5, 2, 16, 64, device="cpu")
    q = torch.zeros(2, 4, 1, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="K must be"):
        mg.mg_paged_append(q, q, Kp, Vp, i)
    with pytest.raises(ValueError, match="rows are"):
        mg.mg_paged_append(q[0], q[0], Kp, Vp, i)
    with pytest.raises(ValueError, match="Kp must be"):
        mg.mg_paged_append(q[0], q[0], Kp[0], Vp, i)
    with pytest.raises(ValueError, match="table must be"):
        mg.mg_paged_resize(i, i, i, i, i, i, i, i, i, page=16)
    for call in (lambda **k: mg.mg_attn_fwd_paged(k["Q"], Kp, Vp, k["t"], i, q, q, causal=True,
                                                  scale=1.0),
                 lambda **k: mg.mg_paged_select(k["Q"], bounds, k["t"], i, k["x"], page=16,
                                                causal=True, first=0, recent=0)):
        with pytest.raises(ValueError, match="must be"):
            call(Q=q[0], t=table, x=bounds)
        with pytest.raises(ValueError, match="must be"):
            call(Q=q, t=i, x=bounds)
    with pytest.raises(ValueError, match="index must be"):
        mg.mg_attn_fwd_paged_sparse(q, Kp, Vp, table, i, i, q, q, causal=True, scale=1.0)
    with pytest.raises(ValueError, match="Kp has shape"):
        mg.mg_attn_fwd_paged(q[..., :32], Kp, Vp, table, i, q, q, causal=True, scale=1.0)
    with pytest.raises(ValueError, match="together"):
        mg.attention_forward_paged(q, Kp, Vp, table, i, causal=True, scale=1.0, keep=3)


# ------------------------------------------------- the tests' plain implementation --
def test_reference_resize_keeps_every_page_once():
    rng = np.random.default_rng(5)
    for _ in range(60):
        B, P, page = int(rng.integers(1, 9)), int(rng.integers(1, 7)), 16
        N = B * P
        order = rng.permutation(N).reshape(B, P)
        lens = rng.integers(0, P * page + 1, B)
        held = np.arange(P) < -(-lens // page)[:, None]
        table = np.where(held, order, -7)
        rest = order[~held]
        count = len(rest) if rng.random() < 0.5 else int(rng.integers(0, len(rest) + 1))
        free = np.concatenate([rest, np.full(N - len(rest), -9)])
        want = rng.integers(0, P * page + 3, B)
        T = int(rng.integers(1, B * P * page))
        owned = set(order[held]) | set(free[:count])
        new_len, left, slot, offset = ref.resize(lens, want, table, free, count, page, T)
        now = [table[b, p] for b in range(B) for p in range(ref.pages(new_len[b], page))]
        assert len(now) + left == len(owned) and set(now) | set(free[:left]) == owned
        for b in range(B):
            assert new_len[b] in (want[b], lens[b])
            rows = slot[offset[b]:offset[b + 1]]
            if want[b] > lens[b] and new_len[b] == want[b]:
                pos = np.arange(lens[b], want[b])
                assert np.array_equal(rows, table[b, pos // page] * page + pos % page)
            else:
                assert np.all(rows == -1)


def test_reference_score_bounds_every_token():
    rng = np.random.default_rng(6)
    N, page, d = 7, 16, 32
    K = rng.standard_normal((page * 5, 1, d))
    Kp, bounds = np.zeros((N, 1, page, d)), np.zeros((N, 1, 2, d))
    slot = np.concatenate([np.arange(page) + page * p for p in (3, 0, 6, 1, 2)])
    ref.append(K, K, Kp, Kp.copy(), bounds, slot, "f32")
    q = rng.standard_normal((4, d))
    s = ref.scores(q, bounds[:, 0], np.array([3, 0, 6, 1, 2, -1, 7]), 7)
    per_page = (K[:, 0] @ q.T).reshape(5, page, 4).max((1, 2))
    assert np.all(s[:5] >= per_page.astype(np.float32)) and np.isnan(s[5:]).all()
    assert ref.select(q, bounds[:, 0], np.array([3, 0, 6, 1, 2, -1, 7]), 7, 3, 0, 1)[-1] == 6
