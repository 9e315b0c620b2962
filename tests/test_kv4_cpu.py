"""Host-side checks of the 4-bit cache (no GPU needed): exported symbols,
sizes, refusals before anything is enqueued, the binding's own checks, and the
tests' plain implementation against the definition."""
import ctypes
import os
import re
import subprocess

import numpy as np
import pytest

import kv4_ref as ref
import paper_2608_01563_amd as mg

vp = ctypes.c_void_p
GOOD = [0x1000 * (k + 1) for k in range(12)]   # aligned, never dereferenced


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(mg.LIB_PATH):
        pytest.fail("libmg.so is not built; run __graft_entry__.build()")
    return mg.load_library()


def test_every_declared_symbol_is_exported(lib):
    with open(mg.KV4_HEADER_PATH) as f:
        text = re.sub(r"/\*.*?\*/", "", f.read(), flags=re.S)
    names = set(re.findall(r"\b(mg_[a-z0-9_]+)\s*\(", text))
    assert {"mg_kv4_append", "mg_kv4_read", "mg_attn_fwd_kv4", "mg_kv4_evict",
            "mg_kv4_cache_bytes", "mg_attn_fwd_kv4_workspace_bytes"} == names
    out = subprocess.run(["nm", "-D", "--defined-only", mg.LIB_PATH], capture_output=True,
                         text=True, check=True).stdout
    exported = {line.split()[-1] for line in out.splitlines() if " T " in line}
    assert names <= exported


@pytest.mark.parametrize("B,H,L,d", [(1, 1, 1, 32), (2, 3, 33, 64), (4, 8, 1000, 128)])
def test_cache_size_is_the_documented_layouts(B, H, L, d):
    assert mg.mg_kv4_cache_bytes(B, H, L, d) == ref.regions(B, H, L, d)[1]


@pytest.mark.parametrize("B,H,L,d", [(0, 1, 1, 32), (1, 0, 1, 32), (1, 1, 0, 32), (1, 1, 1, 48),
                                     (1 << 11, 1 << 10, 1, 32), (1, 1, (1 << 24) + 1, 32),
                                     (1 << 10, 1 << 10, 1 << 11, 32), (-1, -1, 1, 32)])
def test_no_cache_of_bad_sizes(B, H, L, d):
    assert mg.mg_kv4_cache_bytes(B, H, L, d) == 0
    with pytest.raises(ValueError):
        mg.kv4_cache(B, H, L, d)


def test_largest_sizes(lib):
    """Grids of 2^32 threads and more are not launched."""
    for B, H, L, more in ((1 << 19, 1, 32, (1, 0, 0)), (1 << 10, 1 << 9, 1 << 11, (0, 0, 1)),
                          (1 << 3, 1 << 3, 1 << 24, (0, 0, 1))):
        assert mg.mg_kv4_cache_bytes(B, H, L, 32) == ref.regions(B, H, L, 32)[1] > 0
        assert mg.mg_kv4_cache_bytes(B + more[0], H + more[1], L + more[2], 32) == 0
    for call in (append, read):
        # n at its limit: the pointers, which are nobody's, are what is refused
        for n, refused in ((1 << 9, "device"), ((1 << 9) + 1, "rows")):
            assert call(lib, B=1 << 10, H=1 << 9, n=n, L=64) == 1
            assert refused in mg.mg_last_error_detail()


def test_workspace_query():
    f = mg.mg_attn_fwd_kv4_workspace_bytes
    assert f(1, 4, 4, 1, 256, 64) == 0                      # one share a head, no weights
    assert f(64, 32, 8, 1, 4096, 128) == 0                  # enough heads to fill the GPU
    assert f(64, 32, 8, 1, 4096, 128, True) == 64 * 32 * 4096 * 4      # scores
    assert f(64, 32, 8, 9, 4096, 128, True) == 0            # more than 16 rows a head: recomputed
    assert f(1, 8, 1, 1, 1 << 15, 128) > 0                  # shares of the tokens
    for bad in ((1, 5, 4, 1, 256, 64), (1, 0, 4, 1, 256, 64), (1, 4, 4, 0, 256, 64),
                (1, 4, 4, 1, 256, 96), (1 << 10, 1 << 10, 1 << 10, 1 << 12, 256, 64)):
        assert f(*bad) == 0
    assert f(1, 8, 1, 1, 1 << 15, 128, contract=9) == 0


def append(lib, ptrs=GOOD, B=1, H=2, n=3, L=10, d=64, contract=1):
    return lib.mg_kv4_append(*(vp(p) for p in ptrs[:6]), B, H, n, L, d, contract, None)


def read(lib, ptrs=GOOD, B=1, H=2, n=3, L=10, d=64, contract=1):
    return lib.mg_kv4_read(*(vp(p) for p in ptrs[:5]), B, H, n, L, d, contract, None)


@pytest.mark.parametrize("call", [append, read])
@pytest.mark.parametrize("kwargs,status", [
    (dict(B=0), 1), (dict(H=0), 1), (dict(n=0), 1), (dict(L=-1), 1), (dict(d=0), 1),
    (dict(d=96), 2), (dict(contract=3), 1), (dict(contract=-1), 1), (dict(n=(1 << 24) + 1), 1),
    (dict(B=1 << 9, n=1 << 19), 1), (dict(B=1 << 19, H=4), 1)])
def test_move_refuses_bad_sizes(lib, call, kwargs, status):
    assert call(lib, **kwargs) == status
    assert mg.mg_last_error_detail() != ""


def test_move_refuses_bad_pointers(lib):
    for call, need, ints in ((append, (0, 1, 2), (3, 4, 5)), (read, (0, 1, 2), (3, 4))):
        for k in need:
            ptrs = list(GOOD)
            ptrs[k] = 0
            assert call(lib, ptrs) == 1
            ptrs[k] = GOOD[k] + 8
            assert call(lib, ptrs) == 3
    bufs = [ctypes.create_string_buffer(4096) for _ in range(3)]
    host = [(ctypes.addressof(b) + 15) // 16 * 16 for b in bufs]
    assert append(lib, host + [0, 0, 0]) == 1 and "device" in mg.mg_last_error_detail()


def attn(lib, ptrs=GOOD, B=1, Hq=4, H=2, Lq=1, L=64, d=64, scale=0.125, contract=1, ws=0,
         nbytes=0):
    return lib.mg_attn_fwd_kv4(*(vp(p) for p in ptrs[:7]), B, Hq, H, Lq, L, d, 1,
                               ctypes.c_float(scale), contract, vp(ws), nbytes, None)


@pytest.mark.parametrize("kwargs,status", [
    (dict(B=0), 1), (dict(Hq=0), 1), (dict(Hq=3), 1), (dict(Hq=1), 1), (dict(Lq=0), 1),
    (dict(L=0), 1), (dict(d=16), 2), (dict(scale=float("inf")), 1),
    (dict(scale=float("nan")), 1), (dict(contract=7), 1),
    (dict(B=1 << 10, Hq=1 << 10, Lq=1 << 10), 1),
    (dict(L=1 << 15, ws=0x9000, nbytes=16), 4), (dict(L=1 << 15), 4),
    (dict(ptrs=GOOD[:4] + GOOD[4:]), 4)])     # weights: scores need a workspace
def test_attention_refuses_bad_arguments(lib, kwargs, status):
    ptrs = kwargs.pop("ptrs", GOOD[:4] + [0] + GOOD[5:])
    assert attn(lib, ptrs, **kwargs) == status
    assert mg.mg_last_error_detail() != ""


def test_attention_refuses_bad_pointers(lib):
    for k in range(4):
        ptrs = GOOD[:4] + [0] + GOOD[5:]
        ptrs[k] = 0
        assert attn(lib, ptrs) == 1
        ptrs[k] = GOOD[k] + 4
        assert attn(lib, ptrs) == 3


def evict(lib, ptrs=GOOD, B=1, H=2, L=64, d=64, keep=8, recent=2):
    return lib.mg_kv4_evict(*(vp(p) for p in ptrs[:7]), B, H, L, d, keep, recent, None)


@pytest.mark.parametrize("kwargs,status", [
    (dict(B=0), 1), (dict(L=0), 1), (dict(d=33), 2), (dict(keep=0), 1), (dict(keep=65), 1),
    (dict(recent=-1), 1), (dict(recent=9), 1)])
def test_evict_refuses_bad_sizes(lib, kwargs, status):
    assert evict(lib, **kwargs) == status


def test_evict_refuses_bad_pointers(lib):
    same = list(GOOD)
    same[2] = same[0]                      # the cache in place, the weights elsewhere
    assert evict(lib, same) == 1 and "both" in mg.mg_last_error_detail()
    for k in range(6):
        ptrs = list(GOOD)
        ptrs[k] = 0
        assert evict(lib, ptrs) == 1
        ptrs[k] = GOOD[k] + 2
        assert evict(lib, ptrs) == 3


def test_binding_refuses_what_is_not_on_the_gpu(lib):
    import torch
    x = torch.zeros(1, 2, 3, 64, dtype=torch.bfloat16)
    cache = torch.zeros(mg.mg_kv4_cache_bytes(1, 2, 10, 64), dtype=torch.uint8)
    with pytest.raises(ValueError, match="GPU"):
        mg.mg_kv4_append(x, x, cache, L=10)
    with pytest.raises(ValueError, match="GPU"):
        mg.mg_kv4_read(cache, x, x, L=10)
    with pytest.raises(ValueError, match="GPU"):
        mg.mg_attn_fwd_kv4(x, cache, x, torch.zeros(1, 2, 3), H=2, L=10, causal=True, scale=1.0)
    w = torch.zeros(1, 2, 10)
    with pytest.raises(ValueError, match="GPU"):
        mg.mg_kv4_evict(cache, w, torch.zeros(1, 2, 4, dtype=torch.int32),
                        torch.zeros(1, dtype=torch.int32), d=64, recent=1)
    with pytest.raises(ValueError, match="together"):
        mg.mg_kv4_evict(cache, w, torch.zeros(1, 2, 4, dtype=torch.int32),
                        torch.zeros(1, dtype=torch.int32), d=64, recent=1, out_cache=cache)


@pytest.mark.parametrize("d", [32, 64, 128])
def test_reference_layout_round_trip(d):
    rng = np.random.default_rng(d)
    raw = rng.integers(0, 256, ref.regions(2, 3, 70, d)[1]).astype(np.uint8)
    c = ref.Cache.from_bytes(raw, 2, 3, 70, d)
    out = c.to_bytes()
    for at, shape in ref.regions(2, 3, 70, d)[0]:
        n = int(np.prod(shape)) * 4
        assert np.array_equal(out[at:at + n], raw[at:at + n])


def test_reference_codes_are_the_nearest():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((50, 128)).astype(np.float32) * 3 + 1
    code, sc, mn = ref.quantise(x)
    y = ref.values(code, sc, mn)
    s = np.repeat(sc.astype(np.float64), 64, 1)
    # half a step, and at the upper end what the scale's rounding takes away
    assert np.all(np.abs(y - x) <= s * (0.5 + 15 * 2.0 ** -8))
    assert code.max() == 15 and code.min() == 0
