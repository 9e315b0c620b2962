"""ctypes binding of the paged key/value cache (mg_paged.h): argument
marshalling only, in the manner of _binding.py.

Every function checks the tensors it is given, runs on the tensors' own
device (which need not be the current one) and raises MgError on a non-MG_OK
status.  Pools are contiguous tensors [N,H,page,d], bounds [N,H,2,d].
"""
from ._binding import (_alloc_stream, _contract_id, _empty_bytes, _ptr, FAST_BF16,
                       load_library)
from ._kv4 import _call, _elem, _need


def _room(workspace, need, dev, device, stream):
    """(pointer, bytes) of the workspace: the caller's, or one of need() bytes that
    is allocated here (and kept by the third value)."""
    if workspace is None:
        nbytes = need()
        if nbytes == 0:
            return None, 0, None
        workspace = _empty_bytes(nbytes, device, stream)
    elif workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous and on cuda:%d" % dev)
    return workspace.data_ptr(), workspace.nbytes, workspace


# -------------------------------------------------------------------- tables --
def mg_paged_resize_workspace_bytes(B, T):
    return int(load_library().mg_paged_resize_workspace_bytes(B, T))


def mg_paged_resize(key_len, want, table, free_pages, free_count, new_len, new_count, slot,
                    offset, *, page, workspace=None, stream=None):
    """Bring sequences from key_len [B] to want [B] tokens: pages pushed to and
    popped from the stack free_pages [N] of free_count [1] entries, table [B,P]
    written where they grow; new_len [B] (may be key_len), new_count [1] (may be
    free_count), slot [T] of every new row, offset [B+1] of the sequences' rows."""
    import torch
    if table.dim() != 2 or free_pages.dim() != 1 or slot.dim() != 1:
        raise ValueError("table must be [B,P], free_pages [N] and slot [T]")
    B, P = table.shape
    N, T, dev, i32 = free_pages.shape[0], slot.shape[0], table.get_device(), torch.int32
    _need(dev, (("table", table, i32, None), ("key_len", key_len, i32, (B,)),
                ("want", want, i32, (B,)), ("free_pages", free_pages, i32, None),
                ("free_count", free_count, i32, (1,)), ("new_len", new_len, i32, (B,)),
                ("new_count", new_count, i32, (1,)), ("slot", slot, i32, None),
                ("offset", offset, i32, (B + 1,))))
    ws, nbytes, _kept = _room(workspace, lambda: mg_paged_resize_workspace_bytes(B, T), dev,
                              table.device, stream)
    _call(dev, stream, load_library().mg_paged_resize, key_len.data_ptr(), want.data_ptr(),
          table.data_ptr(), free_pages.data_ptr(), free_count.data_ptr(), new_len.data_ptr(),
          new_count.data_ptr(), slot.data_ptr(), offset.data_ptr(), B, page, P, N, T, ws,
          nbytes)


def mg_paged_append(K, V, Kp, Vp, slot, bounds=None, *, contract=FAST_BF16, stream=None):
    """Write rows K, V [T,H,d] to slot [T] of the pools Kp, Vp; bounds
    [N,H,2,d], if given, follow."""
    import torch
    c = _contract_id(contract)
    if K.dim() != 3:
        raise ValueError("K must be [T,H,d]")
    if Kp.dim() != 4:
        raise ValueError("Kp must be [N,H,page,d]")
    rows, pool = K.shape, Kp.shape
    (T, H, d), (N, _, page, _) = rows, pool
    if pool[1] != H or pool[3] != d:
        raise ValueError("Kp has shape %s, rows are [%d,%d,%d]" % (tuple(pool), T, H, d))
    dev, elem = K.get_device(), _elem(c)
    _need(dev, (("K", K, elem, None), ("V", V, elem, rows), ("Kp", Kp, elem, None),
                ("Vp", Vp, elem, pool), ("slot", slot, torch.int32, (T,)),
                ("bounds", bounds, elem, (N, H, 2, d))))
    _call(dev, stream, load_library().mg_paged_append, K.data_ptr(), V.data_ptr(), Kp.data_ptr(),
          Vp.data_ptr(), _ptr(bounds), slot.data_ptr(), T, H, d, page, N, c)


# ----------------------------------------------------------------- attention --
def mg_attn_fwd_paged_workspace_bytes(B, Hq, H, Lq, d, page, P, contract=FAST_BF16):
    return int(load_library().mg_attn_fwd_paged_workspace_bytes(B, Hq, H, Lq, d, page, P,
                                                                _contract_id(contract)))


def mg_attn_fwd_paged_sparse_workspace_bytes(B, Hq, H, Lq, d, page, keep, contract=FAST_BF16):
    return int(load_library().mg_attn_fwd_paged_sparse_workspace_bytes(
        B, Hq, H, Lq, d, page, keep, _contract_id(contract)))


def _attn(Q, Kp, Vp, table, key_len, q_len, index, O, LSE, c, workspace, stream):
    """Checks; sizes and the workspace."""
    import torch
    if Q.dim() != 4 or table.dim() != 2:
        raise ValueError("Q must be [B,Hq,Lq,d] and table [B,P]")
    if Kp.dim() != 4:
        raise ValueError("Kp must be [N,H,page,d]")
    rows, pool = Q.shape, Kp.shape
    (B, Hq, Lq, d), (N, H, page, _), (tables, P) = rows, pool, table.shape
    if pool[3] != d:
        raise ValueError("Kp has shape %s, Q %s" % (tuple(pool), tuple(rows)))
    if tables != B:
        raise ValueError("table has %d rows, Q %d sequences" % (tables, B))
    if index is not None and index.dim() != 4:
        raise ValueError("index must be [B,H,Lq,keep]")
    dev, elem, i32 = Q.get_device(), _elem(c), torch.int32
    _need(dev, (("Q", Q, elem, None), ("Kp", Kp, elem, None), ("Vp", Vp, elem, pool),
                ("O", O, elem, rows), ("LSE", LSE, torch.float32, (B, Hq, Lq)),
                ("table", table, i32, None), ("key_len", key_len, i32, (B,)),
                ("q_len", q_len, i32, (B,))))
    if index is None:
        need = lambda: mg_attn_fwd_paged_workspace_bytes(B, Hq, H, Lq, d, page, P, c)
    else:
        keep = index.shape[3]
        _need(dev, (("index", index, i32, (B, H, Lq, keep)),))
        need = lambda: mg_attn_fwd_paged_sparse_workspace_bytes(B, Hq, H, Lq, d, page, keep, c)
    return (dev, (B, Hq, H, Lq, d, page, P, N),
            _room(workspace, need, dev, Q.device if workspace is None else None, stream))


def mg_attn_fwd_paged(Q, Kp, Vp, table, key_len, O, LSE, q_len=None, *, causal, scale,
                      contract=FAST_BF16, workspace=None, stream=None):
    """Attention of Q [B,Hq,Lq,d] over key_len [B] tokens in the pages of table
    [B,P], into O and LSE [B,Hq,Lq].  `workspace` as for mg_attn_bwd (sized by
    mg_attn_fwd_paged_workspace_bytes; allocated here with torch when None)."""
    c = _contract_id(contract)
    dev, sizes, (ws, nbytes, _kept) = _attn(Q, Kp, Vp, table, key_len, q_len, None, O, LSE, c,
                                            workspace, stream)
    _call(dev, stream, load_library().mg_attn_fwd_paged, Q.data_ptr(), Kp.data_ptr(),
          Vp.data_ptr(), O.data_ptr(), LSE.data_ptr(), table.data_ptr(), key_len.data_ptr(),
          _ptr(q_len), *sizes, 1 if causal else 0, scale, c, ws, nbytes)


def mg_attn_fwd_paged_sparse(Q, Kp, Vp, table, key_len, index, O, LSE, q_len=None, *, causal,
                             scale, contract=FAST_BF16, workspace=None, stream=None):
    """As mg_attn_fwd_paged, where row i of cache head h sees the tokens of pages
    index[b,h,i] ([B,H,Lq,keep], ascending) only."""
    c = _contract_id(contract)
    dev, sizes, (ws, nbytes, _kept) = _attn(Q, Kp, Vp, table, key_len, q_len, index, O, LSE, c,
                                            workspace, stream)
    _call(dev, stream, load_library().mg_attn_fwd_paged_sparse, Q.data_ptr(), Kp.data_ptr(),
          Vp.data_ptr(), O.data_ptr(), LSE.data_ptr(), table.data_ptr(), index.data_ptr(),
          key_len.data_ptr(), _ptr(q_len), *sizes, 1 if causal else 0, index.shape[3], scale, c,
          ws, nbytes)


# ----------------------------------------------------------------- selection --
def mg_paged_select_workspace_bytes(B, Hq, H, Lq, d, page, P, contract=FAST_BF16):
    return int(load_library().mg_paged_select_workspace_bytes(B, Hq, H, Lq, d, page, P,
                                                              _contract_id(contract)))


def mg_paged_select(Q, bounds, table, key_len, index, q_len=None, *, page, causal, first, recent,
                    contract=FAST_BF16, workspace=None, stream=None):
    """For every row of Q [B,Hq,Lq,d] and cache head the pages worth reading, into
    index [B,H,Lq,keep]: the first `first`, the last `recent` and those whose
    bounds [N,H,2,d] promise the largest scores, ascending, -1 behind the last."""
    import torch
    c = _contract_id(contract)
    if Q.dim() != 4 or table.dim() != 2 or bounds.dim() != 4 or index.dim() != 4:
        raise ValueError("Q must be [B,Hq,Lq,d], table [B,P], bounds [N,H,2,d] and index "
                         "[B,H,Lq,keep]")
    (B, Hq, Lq, d), (N, H, _, _) = Q.shape, bounds.shape
    P, keep, i32 = table.shape[1], index.shape[3], torch.int32
    dev, elem = Q.get_device(), _elem(c)
    _need(dev, (("Q", Q, elem, None), ("bounds", bounds, elem, (N, H, 2, d)),
                ("table", table, i32, (B, P)), ("key_len", key_len, i32, (B,)),
                ("q_len", q_len, i32, (B,)), ("index", index, i32, (B, H, Lq, keep))))
    ws, nbytes, _kept = _room(
        workspace, lambda: mg_paged_select_workspace_bytes(B, Hq, H, Lq, d, page, P, c), dev,
        Q.device, stream)
    _call(dev, stream, load_library().mg_paged_select, Q.data_ptr(), bounds.data_ptr(),
          table.data_ptr(), key_len.data_ptr(), _ptr(q_len), index.data_ptr(), B, Hq, H, Lq, d,
          page, P, N, 1 if causal else 0, keep, first, recent, c, ws, nbytes)


# ------------------------------------------------------------ conveniences --
def paged_cache(N, H, page, d, contract=FAST_BF16, bounds=True, device="cuda", stream=None):
    """Allocate pools of N pages with torch: (Kp, Vp, bounds or None)."""
    import torch
    elem = _elem(_contract_id(contract))
    with _alloc_stream(stream):
        Kp, Vp = (torch.empty(N, H, page, d, dtype=elem, device=device) for _ in range(2))
        return Kp, Vp, torch.empty(N, H, 2, d, dtype=elem, device=device) if bounds else None


def attention_forward_paged(Q, Kp, Vp, table, key_len, *, causal, scale, q_len=None, bounds=None,
                            keep=None, first=1, recent=2, contract=None, stream=None):
    """Allocate O and LSE with torch and run attention over the pages, over the
    `keep` best pages of every row only if that is given (with bounds); returns
    (O, LSE)."""
    import torch
    c = _contract_id(contract) if contract is not None else (
        FAST_BF16 if Q.dtype == torch.bfloat16 else 0)
    if (keep is None) != (bounds is None):
        raise ValueError("give keep and bounds together")
    if Q.dim() != 4 or Kp.dim() != 4:
        raise ValueError("Q must be [B,Hq,Lq,d] and Kp [N,H,page,d]")
    kw = dict(causal=causal, contract=c, stream=stream)
    with _alloc_stream(stream):
        O = torch.empty_like(Q)
        LSE = torch.empty(Q.shape[:3], dtype=torch.float32, device=Q.device)
        if keep is not None:
            index = torch.empty(Q.shape[0], Kp.shape[1], Q.shape[2], keep, dtype=torch.int32,
                                device=Q.device)
    if keep is None:
        mg_attn_fwd_paged(Q, Kp, Vp, table, key_len, O, LSE, q_len, scale=scale, **kw)
    else:
        mg_paged_select(Q, bounds, table, key_len, index, q_len, page=Kp.shape[2], first=first,
                        recent=recent, **kw)
        mg_attn_fwd_paged_sparse(Q, Kp, Vp, table, key_len, index, O, LSE, q_len, scale=scale, **kw)
    return O, LSE
