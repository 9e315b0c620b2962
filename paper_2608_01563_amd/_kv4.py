"""ctypes binding of the 4-bit key/value cache (mg_kv4.h): argument
marshalling only, in the manner of _binding.py.

Every function checks the tensors it is given, runs on the tensors' own
device (which need not be the current one) and raises MgError on a non-MG_OK
status.  A cache is a uint8 tensor of exactly mg_kv4_cache_bytes(B, H, L, d) bytes.
"""
import functools

from ._binding import (_alloc_stream, _check, _contract_id, _empty_bytes, _ptr, FAST_BF16,
                       load_library)


def _elem(contract):
    import torch
    return torch.bfloat16 if contract == FAST_BF16 else torch.float32


def _need(dev, named):
    """Every (name, tensor, dtype, shape) of `named` that is not None must be a
    contiguous tensor of that dtype and shape (None: any) on GPU `dev`."""
    if dev < 0:
        raise ValueError("%s must be a GPU tensor" % named[0][0])
    for name, t, dtype, shape in named:
        if t is None or (t.get_device() == dev and t.dtype is dtype and
                         (shape is None or t.shape == shape) and t.is_contiguous()):
            continue
        if not t.is_cuda:
            raise ValueError("%s must be a GPU tensor" % name)
        if t.get_device() != dev:
            raise ValueError("%s is on %s, the others on cuda:%d" % (name, t.device, dev))
        if t.dtype is not dtype:
            raise ValueError("%s has dtype %s, expected %s" % (name, t.dtype, dtype))
        if shape is not None and tuple(t.shape) != tuple(shape):
            raise ValueError("%s has shape %s, expected %s" % (name, tuple(t.shape), tuple(shape)))
        raise ValueError("%s must be contiguous" % name)


def _need_room(cache, B, H, L, d):
    """The cache must be one of these sizes: in a larger one another layout lies."""
    need = mg_kv4_cache_bytes(B, H, L, d)   # 0 for bad sizes: the library says why
    if need and cache.numel() != need:
        raise ValueError("the cache has %d bytes, B=%d H=%d L=%d d=%d needs %d"
                         % (cache.numel(), B, H, L, d, need))


def _call(dev, stream, function, *args):
    """function(*args, stream handle) with the tensors' GPU the current one; a
    given stream must be that GPU's."""
    import torch
    if stream is not None and stream.device.index != dev:
        raise ValueError("the stream belongs to %s, the tensors to cuda:%d" % (stream.device, dev))
    handle = torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream
    if dev == torch.cuda.current_device():
        _check(function(*args, handle))
    else:
        with torch.cuda.device(dev):
            _check(function(*args, handle))


@functools.lru_cache(maxsize=256)
def mg_kv4_cache_bytes(B, H, L, d):
    """Bytes of a cache of B sequences, H heads, L tokens; 0 for invalid sizes."""
    return int(load_library().mg_kv4_cache_bytes(int(B), int(H), int(L), int(d)))


def _move(K, V, cache, start, count, L, contract, weight=None):
    import torch
    if K.dim() != 4:
        raise ValueError("K must be [B,H,n,d]")
    B, H, n, d = K.shape
    dev, elem = K.get_device(), _elem(contract)
    _need(dev, (("K", K, elem, K.shape), ("V", V, elem, K.shape),
                ("cache", cache, torch.uint8, None), ("start", start, torch.int32, (B,)),
                ("count", count, torch.int32, (B,)), ("weight", weight, torch.float32, (B, H, L))))
    _need_room(cache, B, H, L, d)
    return dev, B, H, n, d


def mg_kv4_append(K, V, cache, start=None, count=None, *, L, weight=None, contract=FAST_BF16,
                  stream=None):
    """Write rows j < count[b] of K, V [B,H,n,d] as tokens start[b] + j of a
    cache with room for L tokens (count None: n; start None: 0); `weight`
    [B,H,L], if given, is cleared for them."""
    c = _contract_id(contract)
    dev, B, H, n, d = _move(K, V, cache, start, count, L, c, weight)
    _call(dev, stream, load_library().mg_kv4_append, K.data_ptr(), V.data_ptr(),
          cache.data_ptr(), _ptr(weight), _ptr(start), _ptr(count), B, H, n, L, d, c)


def mg_kv4_read(cache, K, V, start=None, count=None, *, L, contract=FAST_BF16, stream=None):
    """Read tokens start[b] + j, j < count[b], back into rows j of K, V
    [B,H,n,d]; other rows are left as they were."""
    c = _contract_id(contract)
    dev, B, H, n, d = _move(K, V, cache, start, count, L, c)
    _call(dev, stream, load_library().mg_kv4_read, cache.data_ptr(), K.data_ptr(), V.data_ptr(),
          _ptr(start), _ptr(count), B, H, n, L, d, c)


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
    c = _contract_id(contract)
    if Q.dim() != 4:
        raise ValueError("Q must be [B,Hq,Lq,d]")
    B, Hq, Lq, d = Q.shape
    dev, elem = Q.get_device(), _elem(c)
    _need(dev, (("Q", Q, elem, Q.shape), ("O", O, elem, Q.shape),
                ("LSE", LSE, torch.float32, Q.shape[:3]), ("cache", cache, torch.uint8, None),
                ("key_len", key_len, torch.int32, (B,)), ("q_len", q_len, torch.int32, (B,)),
                ("weight", weight, torch.float32, (B, H, L))))
    _need_room(cache, B, H, L, d)
    if workspace is None:
        need = mg_attn_fwd_kv4_workspace_bytes(B, Hq, H, Lq, L, d, weight is not None, c)
        if need > 0:
            workspace = _empty_bytes(need, Q.device, stream)
    nbytes = 0
    if workspace is not None:
        if workspace.get_device() != dev or not workspace.is_contiguous():
            raise ValueError("workspace must be contiguous and on cuda:%d" % dev)
        nbytes = workspace.numel() * workspace.element_size()
    _call(dev, stream, load_library().mg_attn_fwd_kv4, Q.data_ptr(), cache.data_ptr(),
          O.data_ptr(), LSE.data_ptr(), _ptr(weight), _ptr(key_len), _ptr(q_len), B, Hq, H, Lq,
          L, d, 1 if causal else 0, scale, c, _ptr(workspace), nbytes)


def mg_kv4_evict(cache, weight, index, new_len, key_len=None, *, d, recent, out_cache=None,
                 out_weight=None, stream=None):
    """Cut sequences of weight [B,H,L] to index.shape[2] tokens, the last
    `recent` and those of largest weight, in place or into out_cache and
    out_weight; index [B,H,keep] gets where they were (-1 behind the last) and
    new_len [B] how many stay (it may be key_len itself)."""
    import torch
    if weight.dim() != 3 or index.dim() != 3:
        raise ValueError("weight must be [B,H,L] and index [B,H,keep]")
    B, H, L = weight.shape
    keep, dev = index.shape[2], weight.get_device()
    if (out_cache is None) != (out_weight is None):
        raise ValueError("give out_cache and out_weight together")
    if out_cache is None:
        out_cache, out_weight = cache, weight
    _need(dev, (("weight", weight, torch.float32, (B, H, L)),
                ("out_weight", out_weight, torch.float32, (B, H, L)),
                ("index", index, torch.int32, (B, H, keep)),
                ("new_len", new_len, torch.int32, (B,)),
                ("key_len", key_len, torch.int32, (B,)),
                ("cache", cache, torch.uint8, None), ("out_cache", out_cache, torch.uint8, None)))
    _need_room(cache, B, H, L, d)
    _need_room(out_cache, B, H, L, d)
    _call(dev, stream, load_library().mg_kv4_evict, cache.data_ptr(), weight.data_ptr(),
          out_cache.data_ptr(), out_weight.data_ptr(), index.data_ptr(), new_len.data_ptr(),
          _ptr(key_len), B, H, L, d, keep, recent)


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
