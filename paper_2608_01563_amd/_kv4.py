"""ctypes binding of the 4-bit key/value cache (mg_kv4.h): argument
marshalling only, in the manner of _binding.py.

Every function checks the tensors it is given, runs on the tensors' own
device (which need not be the current one) and raises MgError on a non-MG_OK
status.  A cache is a uint8 tensor of mg_kv4_cache_bytes(B, H, L, d) bytes.
"""
import contextlib

from ._binding import (_alloc_stream, _check, _contract_id, _empty_bytes, _ptr,
                       _stream_handle, FAST_BF16, load_library)


def _elem(contract):
    import torch
    return torch.bfloat16 if contract == FAST_BF16 else torch.float32


def _need(name, t, dtype, shape, device):
    """`t` must be a contiguous tensor of `dtype` and `shape` (None: any) on `device`."""
    if not t.is_cuda:
        raise ValueError("%s must be a GPU tensor" % name)
    if t.device != device:
        raise ValueError("%s is on %s, the others on %s" % (name, t.device, device))
    if t.dtype != dtype:
        raise ValueError("%s has dtype %s, expected %s" % (name, t.dtype, dtype))
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError("%s has shape %s, expected %s" % (name, tuple(t.shape), tuple(shape)))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)


def _need_cache(name, cache, B, H, L, d, device):
    import torch
    _need(name, cache, torch.uint8, None, device)
    need = mg_kv4_cache_bytes(B, H, L, d)
    if need == 0:   # let the library say why
        return
    if cache.numel() < need:
        raise ValueError("%s has %d bytes, a cache of B=%d H=%d L=%d d=%d needs %d"
                         % (name, cache.numel(), B, H, L, d, need))


def _need_lens(named, B, device):
    import torch
    for name, t in named:
        if t is not None:
            _need(name, t, torch.int32, (B,), device)


@contextlib.contextmanager
def _on(device, stream):
    """Make `device` the current one for the launch; a given stream must be its."""
    import torch
    if stream is not None and stream.device != device:
        raise ValueError("the stream belongs to %s, the tensors to %s" % (stream.device, device))
    if device.index == torch.cuda.current_device():
        yield
    else:
        with torch.cuda.device(device):
            yield


def mg_kv4_cache_bytes(B, H, L, d):
    """Bytes of a cache of B sequences, H heads, L tokens; 0 for invalid sizes."""
    return int(load_library().mg_kv4_cache_bytes(int(B), int(H), int(L), int(d)))


def _move(K, V, cache, start, count, L, contract):
    if K.dim() != 4:
        raise ValueError("K must be [B,H,n,d]")
    B, H, n, d = K.shape
    for what, t in (("K", K), ("V", V)):
        _need(what, t, _elem(contract), K.shape, K.device)
    _need_cache("cache", cache, B, H, L, d, K.device)
    _need_lens((("start", start), ("count", count)), B, K.device)
    return B, H, n, d


def mg_kv4_append(K, V, cache, start=None, count=None, *, L, weight=None, contract=FAST_BF16,
                  stream=None):
    """Write rows j < count[b] of K, V [B,H,n,d] as tokens start[b] + j of a
    cache with room for L tokens (count None: n; start None: 0); `weight`
    [B,H,L], if given, is cleared for them."""
    import torch
    lib, c = load_library(), _contract_id(contract)
    B, H, n, d = _move(K, V, cache, start, count, L, c)
    if weight is not None:
        _need("weight", weight, torch.float32, (B, H, L), K.device)
    with _on(K.device, stream):
        _check(lib.mg_kv4_append(_ptr(K), _ptr(V), _ptr(cache), _ptr(weight), _ptr(start),
                                 _ptr(count), B, H, n, int(L), d, c, _stream_handle(stream)))


def mg_kv4_read(cache, K, V, start=None, count=None, *, L, contract=FAST_BF16, stream=None):
    """Read tokens start[b] + j, j < count[b], back into rows j of K, V
    [B,H,n,d]; other rows are left as they were."""
    lib, c = load_library(), _contract_id(contract)
    B, H, n, d = _move(K, V, cache, start, count, L, c)
    with _on(K.device, stream):
        _check(lib.mg_kv4_read(_ptr(cache), _ptr(K), _ptr(V), _ptr(start), _ptr(count), B, H, n,
                               int(L), d, c, _stream_handle(stream)))


def mg_attn_fwd_kv4_workspace_bytes(B, Hq, H, Lq, L, d, weights=False, contract=FAST_BF16):
    return int(load_library().mg_attn_fwd_kv4_workspace_bytes(
        B, Hq, H, Lq, L, d, int(bool(weights)), _contract_id(contract)))


def mg_attn_fwd_kv4(Q, cache, O, LSE, key_len=None, q_len=None, *, H, L, causal, scale,
                    weight=None, contract=FAST_BF16, workspace=None, stream=None):
    """Attention of Q [B,Hq,Lq,d] over a cache of H heads and room for L tokens
    into O and LSE [B,Hq,Lq]; `weight` [B,H,L], if given, grows by the tokens'
    probabilities.  `workspace` as for mg_attn_bwd (sized by
    mg_attn_fwd_kv4_workspace_bytes; allocated here with torch when None)."""
    import torch
    lib, c = load_library(), _contract_id(contract)
    if Q.dim() != 4:
        raise ValueError("Q must be [B,Hq,Lq,d]")
    B, Hq, Lq, d = Q.shape
    dev = Q.device
    for name, t in (("Q", Q), ("O", O)):
        _need(name, t, _elem(c), Q.shape, dev)
    _need("LSE", LSE, torch.float32, Q.shape[:3], dev)
    _need_cache("cache", cache, B, H, L, d, dev)
    _need_lens((("key_len", key_len), ("q_len", q_len)), B, dev)
    if weight is not None:
        _need("weight", weight, torch.float32, (B, H, L), dev)
    with _on(dev, stream):
        if workspace is None:
            need = mg_attn_fwd_kv4_workspace_bytes(B, Hq, H, Lq, L, d, weight is not None, c)
            if need > 0:
                workspace = _empty_bytes(need, dev, stream)
        nbytes = 0
        if workspace is not None:
            if workspace.device != dev or not workspace.is_contiguous():
                raise ValueError("workspace must be contiguous and on %s" % dev)
            nbytes = workspace.numel() * workspace.element_size()
        _check(lib.mg_attn_fwd_kv4(_ptr(Q), _ptr(cache), _ptr(O), _ptr(LSE), _ptr(weight),
                                   _ptr(key_len), _ptr(q_len), B, Hq, int(H), Lq, int(L), d,
                                   int(bool(causal)), float(scale), c, _ptr(workspace), nbytes,
                                   _stream_handle(stream)))


def mg_kv4_evict(cache, weight, index, new_len, key_len=None, *, d, recent, out_cache=None,
                 out_weight=None, stream=None):
    """Cut sequences of weight [B,H,L] to index.shape[2] tokens, the last
    `recent` and those of largest weight, in place or into out_cache and
    out_weight; index [B,H,keep] gets where they were (-1 behind the last) and
    new_len [B] how many stay (it may be key_len itself)."""
    import torch
    lib = load_library()
    if weight.dim() != 3 or index.dim() != 3:
        raise ValueError("weight must be [B,H,L] and index [B,H,keep]")
    B, H, L = weight.shape
    keep, dev = index.shape[2], weight.device
    if (out_cache is None) != (out_weight is None):
        raise ValueError("give out_cache and out_weight together")
    if out_cache is None:
        out_cache, out_weight = cache, weight
    for name, t in (("weight", weight), ("out_weight", out_weight)):
        _need(name, t, torch.float32, (B, H, L), dev)
    _need("index", index, torch.int32, (B, H, keep), dev)
    _need("new_len", new_len, torch.int32, (B,), dev)
    for name, t in (("cache", cache), ("out_cache", out_cache)):
        _need_cache(name, t, B, H, L, d, dev)
    _need_lens((("key_len", key_len),), B, dev)
    with _on(dev, stream):
        _check(lib.mg_kv4_evict(_ptr(cache), _ptr(weight), _ptr(out_cache), _ptr(out_weight),
                                _ptr(index), _ptr(new_len), _ptr(key_len), B, H, L, int(d), keep,
                                int(recent), _stream_handle(stream)))


# ------------------------------------------------------------ conveniences --
def kv4_cache(B, H, L, d, device="cuda", stream=None):
    """Allocate a cache with torch; ValueError for sizes it cannot have."""
    need = mg_kv4_cache_bytes(B, H, L, d)
    if need == 0:
        raise ValueError("no cache of B=%d H=%d L=%d d=%d" % (B, H, L, d))
    return _empty_bytes(need, device, stream)


def attention_forward_kv4(Q, cache, *, H, L, causal, scale, key_len=None, q_len=None, weight=None,
                          contract=None, stream=None):
    """Allocate O and LSE with torch and run attention over the cache; returns
    (O, LSE)."""
    import torch
    c = _contract_id(contract) if contract is not None else (
        FAST_BF16 if Q.dtype == torch.bfloat16 else 0)
    with _alloc_stream(stream):
        O = torch.empty_like(Q)
        LSE = torch.empty(Q.shape[:3], dtype=torch.float32, device=Q.device)
    mg_attn_fwd_kv4(Q, cache, O, LSE, key_len, q_len, H=H, L=L, causal=causal, scale=scale,
                    weight=weight, contract=c, stream=stream)
    return O, LSE
