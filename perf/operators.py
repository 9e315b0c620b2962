"""The operators of the 4-bit key/value cache whose speed counts for a user of
this library, each in its plain form (elementary torch operations in 32 bits)
and through the library's entry points.

A case is one pass: tokens written into a cache and read back as the values
they then stand for (`mg_kv4_append`, `mg_kv4_read`), attention of a few or many
query rows over the cache (`mg_attn_fwd_kv4`, with or without the keys'
accumulated attention weights), or the eviction of the tokens with the least
weight (`mg_kv4_evict`).

A token's K (and V) row of one head is held as 4-bit codes with a scale and a
minimum (bf16 each) for every group of min(d, 64) channels:

  min = bf16(min x), scale = bf16((max x - min x) / 15),
  code = clamp(round((x - min) / scale), 0, 15), value = scale * code + min

(rounding to nearest even; code 0 where the scale is 0).
"""
import math

import torch

own = False


# ---------------------------------------------------------------------- cases --
def _append(name, B, H, n, L, d, contract, ragged):
    """n new tokens a sequence into a cache of L; ragged: every sequence has
    its own start and its own number of new tokens (at most n)."""
    return {"name": name, "kind": "append", "B": B, "H": H, "n": n, "L": L, "d": d,
            "contract": contract, "ragged": ragged}


def _evict(name, B, H, L, d, keep, recent, ragged):
    """Sequences of up to L tokens cut to `keep`, the last `recent` among them."""
    return {"name": name, "kind": "evict", "B": B, "H": H, "L": L, "d": d, "keep": keep,
            "recent": recent, "ragged": ragged}


def _attn(name, B, Hq, H, Lq, L, d, contract, ragged, weights=False, empty=False):
    """Lq query rows (the last tokens of their sequence, causal) of Hq heads
    over a cache of H heads; ragged: caches filled to a quarter and more, and
    for Lq > 1 sequences with fewer rows; empty: the first sequence holds
    nothing."""
    return {"name": name, "kind": "attn", "B": B, "Hq": Hq, "H": H, "Lq": Lq, "L": L, "d": d,
            "contract": contract, "ragged": ragged, "weights": weights, "empty": empty}


def listed():
    return [
        # a decode step of a served batch: one token a sequence joins its cache
        _append("append tokens bf16", 64, 8, 1, 2048, 128, "fast_bf16", True),
        # prompts of a batch enter an empty cache, padded to the longest
        _append("append prompts bf16", 4, 8, 8192, 8192, 128, "fast_bf16", True),
        # an odd-length sequence in full precision, six heads of 64
        _append("append ragged f32", 2, 6, 1500, 1601, 64, "strict_f32", True),
        # chat sequences cut to a quarter once they reach 4,096 tokens
        _evict("evict chat", 8, 8, 4096, 128, 1024, 256, False),
        # long documents, of different lengths
        _evict("evict long", 2, 8, 32768, 128, 8192, 500, True),
        # the smallest decode step: launches and latency
        _attn("decode tiny bf16", 1, 4, 4, 1, 256, 64, "fast_bf16", False),
        # an ordinary served batch with grouped heads, the weights kept for eviction
        _attn("decode grouped weights bf16", 16, 32, 8, 1, 4096, 128, "fast_bf16", True, True),
        # a long-context batch, the largest cache
        _attn("decode long bf16", 8, 32, 8, 1, 32768, 128, "fast_bf16", True),
        # full-precision queries, a head of its own each, odd length
        _attn("decode ragged f32", 2, 6, 6, 1, 1500, 64, "strict_f32", True),
        # seven drafted tokens a sequence scored at once
        _attn("draft rows bf16", 8, 32, 8, 7, 4001, 128, "fast_bf16", True),
        # a chunk of a long prompt over what the cache holds so far
        _attn("prefill chunk bf16", 2, 32, 8, 2048, 8192, 128, "fast_bf16", False),
        # a padded batch of prompts whose weights start the eviction's account
        _attn("prefill weights bf16", 4, 16, 4, 1000, 1000, 64, "fast_bf16", True, True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    what = rng.random()
    d = rng.choice((32, 64, 128, 128))
    contract = rng.choice(("fast_bf16", "fast_bf16", "strict_f32"))
    B = _log(rng, 1, 32)
    H = rng.choice((1, 2, 4, 6, 8))
    if what < 0.2:
        n = rng.choice((1, _log(rng, 1, 4096)))
        c = _append("", B, H, n, n + _log(rng, 1, 4096), d, contract, rng.random() < 0.7)
        while c["B"] * c["H"] * c["n"] * c["d"] > 3e7:
            c["B"] = max(1, c["B"] // 2)
            c["n"] = max(1, c["n"] - c["n"] // 8)
    elif what < 0.4:
        L = _log(rng, 40, 32768)
        keep = max(2, int(L * rng.uniform(0.1, 0.9)))
        c = _evict("", B, H, L, d, keep, int(keep * rng.uniform(0.0, 1.0)), rng.random() < 0.7)
        while c["B"] * c["H"] * c["L"] > 5e5 and c["B"] > 1:
            c["B"] = c["B"] // 2
    else:
        Lq = rng.choice((1, 1, 1, rng.randint(2, 9), _log(rng, 10, 1500)))
        L = max(Lq, _log(rng, 16, 32768 if Lq < 10 else 6000))
        c = _attn("", B, H * rng.choice((1, 2, 4, 8)), H, Lq, L, d, contract, rng.random() < 0.7,
                  rng.random() < 0.3, rng.random() < 0.1)
        most = 6e9 if contract == "fast_bf16" else 1.5e9   # pairs * d
        while c["B"] > 1 and (c["B"] * c["Hq"] * c["Lq"] * c["L"] * c["d"] > most or
                              c["B"] * c["H"] * c["L"] * c["d"] > 2e8):
            c["B"] = c["B"] // 2
        while c["Lq"] > 9 and c["Hq"] * c["Lq"] * c["L"] * c["d"] > most:
            c["Lq"] = c["Lq"] - c["Lq"] // 8
            c["L"] = max(c["Lq"], c["L"] - c["L"] // 8)
    return {k: v for k, v in c.items() if k != "name"}


# ------------------------------------------------------------- the cache's parts --
def _groups(d):
    return max(1, d // 64)


def _quantise(x):
    """Codes (uint8) and the groups' scales and minima (f32 holding bf16 values)."""
    ng = _groups(x.shape[-1])
    x = x.float().unflatten(-1, (ng, -1))
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    mn = lo.bfloat16().float()
    # a quotient of tensors: division by a number may multiply by its rounded inverse
    sc = ((hi - lo) / torch.full_like(hi, 15.0)).bfloat16().float()
    # in 64 bits: a quotient next to a border must fall on its own side of it
    q = (x.double() - mn.double()) / torch.where(sc > 0, sc, 1.0).double()
    codes = torch.where(sc > 0, q.round().clamp(0, 15), 0.0).to(torch.uint8)
    return codes.flatten(-2), sc.squeeze(-1), mn.squeeze(-1)


def _values(codes, sc, mn):
    ng = sc.shape[-1]
    c = codes.float().unflatten(-1, (ng, -1))
    return (c * sc.unsqueeze(-1) + mn.unsqueeze(-1)).flatten(-2)


def _bits(t):
    return t.bfloat16().view(torch.int16).to(torch.int64) & 0xffff


def _words(nibbles, dim):
    """Eight codes along `dim` as one 32-bit word, the first in the lowest bits."""
    shape = [1] * nibbles.dim()
    shape[dim] = 8
    shift = (4 * torch.arange(8, device=nibbles.device)).reshape(shape)
    return (nibbles.to(torch.int64) << shift).sum(dim).to(torch.int32)


def _region(t):
    raw = t.flatten().clone().view(torch.uint8)
    return torch.nn.functional.pad(raw, (0, -raw.numel() % 256))


def _pack(k, v, L):
    """The cache's bytes from (codes, scale, min) of K and V, each [B,H,L,...]:
    K's words, V's words, K's and V's group words, every region a multiple of
    256 bytes, tokens padded to a multiple of 32."""
    pad = -L % 32
    (kc, ks, km), (vc, vs, vm) = ([torch.nn.functional.pad(t, (0, 0, 0, pad)) for t in x]
                                  for x in (k, v))
    B, H, Lp, d = kc.shape
    wide = min(4, d // 16)
    kw = _words(kc.reshape(B, H, Lp, d // 32, 4, 8), 5).transpose(3, 4)
    vw = _words(vc.reshape(B, H, Lp // 8, 8, d), 3)
    vw = vw.reshape(B, H, Lp // 8, d // 16 // wide, wide, 16).transpose(4, 5)
    params = [((_bits(s) << 16) | _bits(m)).to(torch.int32) for s, m in ((ks, km), (vs, vm))]
    return torch.cat([_region(t) for t in (kw, vw, *params)])


# ---------------------------------------------------------------------- inputs --
def _dtype(c):
    return torch.bfloat16 if c.get("contract") == "fast_bf16" else torch.float32


def _rows(g, c, n):
    """K or V rows: channels of different size, some of them large and off zero."""
    x = torch.randn(c["B"], c["H"], n, c["d"], generator=g, device="cuda")
    size = torch.exp(0.5 * torch.randn(c["H"], 1, c["d"], generator=g, device="cuda"))
    off = torch.randn(c["H"], 1, c["d"], generator=g, device="cuda")
    return x * size + 0.5 * off


def _ints(g, lo, hi, B):
    return torch.randint(lo, max(hi, lo) + 1, (B,), generator=g, device="cuda", dtype=torch.int32)


def _inputs(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    B, H, L, d = c["B"], c["H"], c["L"], c["d"]
    s = {"case": c}
    if c["kind"] == "append":
        n = c["n"]
        s["K"], s["V"] = (_rows(g, c, n).to(_dtype(c)) for _ in range(2))
        s["count"] = _ints(g, max(1, n // 4), n, B) if c["ragged"] else None
        s["start"] = _ints(g, 0, L - n, B) if c["ragged"] else None
        s["weight"] = torch.rand(B, H, L, generator=g, device="cuda")
        return s
    k, v = _quantise(_rows(g, c, L)), _quantise(_rows(g, c, L))
    s["k"], s["v"] = k, v
    if c["kind"] == "evict":
        s["key_len"] = _ints(g, max(1, L // 4), L, B) if c["ragged"] else None
        # heavy-tailed, as attention leaves them, with many equal small values
        w = torch.exp(2.0 * torch.randn(B, H, L, generator=g, device="cuda") - 2.0)
        s["weight"] = torch.where(w < 0.05, 0.03125, w)
        return s
    Lq = c["Lq"]
    s["Q"] = torch.randn(B, c["Hq"], Lq, d, generator=g, device="cuda").to(_dtype(c))
    s["key_len"] = _ints(g, max(Lq, L // 4), L, B) if c["ragged"] else None
    s["q_len"] = _ints(g, max(1, Lq // 2), Lq, B) if c["ragged"] and Lq > 1 else None
    if c["empty"]:
        s["key_len"] = torch.full((B,), L, dtype=torch.int32, device="cuda") \
            if s["key_len"] is None else s["key_len"]
        s["key_len"][0] = 0
        if s["q_len"] is not None:
            s["q_len"][0] = 0
    s["weight"] = torch.rand(B, H, L, generator=g, device="cuda") if c["weights"] else None
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    B, H, L, d = case["B"], case["H"], case["L"], case["d"]
    none = torch.zeros(B, H, L, d, dtype=torch.uint8, device="cuda")
    zero = torch.zeros(B, H, L, _groups(d), device="cuda")
    if case["kind"] == "append":   # an empty cache, and where the rows are read back to
        s["cache"] = _pack((none, zero, zero), (none, zero, zero), L)
        s["outK"], s["outV"] = torch.zeros_like(s["K"]), torch.zeros_like(s["V"])
    else:
        # the same cache twice: as the library holds it, and a code to a byte
        # with its scales and minima (k, v), which the plain form reads
        s["cache"] = _pack(s["k"], s["v"], L)
    if case["kind"] == "evict":
        keep = case["keep"]
        s["out_cache"] = _pack((none, zero, zero), (none, zero, zero), L)
        s["out_weight"] = torch.zeros_like(s["weight"])
        s["index"] = torch.zeros(B, H, keep, dtype=torch.int32, device="cuda")
        s["new_len"] = torch.zeros(B, dtype=torch.int32, device="cuda")
        s["outK"], s["outV"] = (torch.zeros(B, H, keep, d, device="cuda") for _ in range(2))
    if case["kind"] == "attn":
        s["O"] = torch.empty_like(s["Q"])
        s["LSE"] = torch.empty(s["Q"].shape[:3], device="cuda")
    return s


# ---------------------------------------------------------------- plain forms --
def _lengths(s, name, full):
    B = s["case"]["B"]
    return torch.full((B,), full, device="cuda") if s[name] is None else s[name].to(torch.int64)


def _plain_append(s):
    c = s["case"]
    count, start = _lengths(s, "count", c["n"]), _lengths(s, "start", 0)
    there = (torch.arange(c["n"], device="cuda") < count[:, None])[:, None, :, None]
    K, V = (torch.where(there, _values(*_quantise(x)), 0.0).to(x.dtype) for x in (s["K"], s["V"]))
    j = torch.arange(c["L"], device="cuda")
    new = (j >= start[:, None]) & (j < (start + count)[:, None])
    s["weight"].masked_fill_(new[:, None, :], 0.0)
    return {"K": K, "V": V, "weight": s["weight"]}


def _plain_evict(s):
    c = s["case"]
    L, keep, recent = c["L"], c["keep"], c["recent"]
    n = _lengths(s, "key_len", L)[:, None, None]
    j = torch.arange(L, device="cuda")
    w = torch.where(j >= n - recent, math.inf, s["weight"]).masked_fill(j >= n, -math.inf)
    # the stable order puts equal weights by their index
    chosen = torch.sort(w, dim=2, descending=True, stable=True).indices[:, :, :keep]
    left = torch.minimum(n, torch.tensor(keep, device="cuda"))
    gone = torch.arange(keep, device="cuda") >= left
    index = torch.sort(chosen.masked_fill(gone, L), dim=2).values
    at = index.clamp(max=L - 1)

    def take(t):
        return t.gather(2, at[..., None].expand(*at.shape, t.shape[-1]))

    K, V = (_values(*(take(t) for t in x)).masked_fill(gone[..., None], 0.0)
            for x in (s["k"], s["v"]))
    weight = torch.zeros_like(s["weight"])
    weight[:, :, :keep] = s["weight"].gather(2, at).masked_fill(gone, 0.0)
    return {"K": K, "V": V, "weight": weight, "new_len": left.flatten().to(torch.int32),
            "index": index.masked_fill(gone, -1).to(torch.int32)}


def _plain_attn(s):
    c = s["case"]
    B, Hq, H, Lq, L, d = (c[k] for k in ("B", "Hq", "H", "Lq", "L", "d"))
    n, rows = (_lengths(s, k, f)[:, None, None, None] for k, f in (("key_len", L), ("q_len", Lq)))
    K, V = _values(*s["k"]), _values(*s["v"])
    Q = s["Q"].float().reshape(B, H, Hq // H * Lq, d)
    S = torch.matmul(Q, K.transpose(2, 3).contiguous()).reshape(B, Hq, Lq, L) / math.sqrt(d)
    i = torch.arange(Lq, device="cuda")[:, None]
    j = torch.arange(L, device="cuda")
    S = S.masked_fill(~((j < n) & (j <= i + n - rows) & (i < rows)), -math.inf)
    top = S.amax(3, keepdim=True)
    P = torch.exp(S - torch.where(top == -math.inf, 0.0, top))
    sums = P.sum(3, keepdim=True)
    P = P / torch.where(sums > 0, sums, 1.0)
    O = torch.matmul(P.reshape(B, H, Hq // H * Lq, L), V).reshape(B, Hq, Lq, d)
    LSE = torch.where(sums > 0, top + torch.log(sums), -math.inf).squeeze(3)
    out = {"O": O.to(s["Q"].dtype), "LSE": LSE}
    if s["weight"] is not None:
        s["weight"] += P.reshape(B, H, Hq // H * Lq, L).sum(2)
        out["weight"] = s["weight"]
    return out


# ------------------------------------------------------- the library's entry points --
def _own_append(s):
    import paper_2608_01563_amd as mg
    L, contract = s["case"]["L"], s["case"]["contract"]
    mg.mg_kv4_append(s["K"], s["V"], s["cache"], s["start"], s["count"], L=L, weight=s["weight"],
                     contract=contract)
    mg.mg_kv4_read(s["cache"], s["outK"], s["outV"], s["start"], s["count"], L=L,
                   contract=contract)
    return {"K": s["outK"], "V": s["outV"], "weight": s["weight"]}


def _own_evict(s):
    import paper_2608_01563_amd as mg
    c = s["case"]
    mg.mg_kv4_evict(s["cache"], s["weight"], s["index"], s["new_len"], s["key_len"], d=c["d"],
                    recent=c["recent"], out_cache=s["out_cache"], out_weight=s["out_weight"])
    mg.mg_kv4_read(s["out_cache"], s["outK"], s["outV"], None, s["new_len"], L=c["L"],
                   contract="strict_f32")
    return {"K": s["outK"], "V": s["outV"], "weight": s["out_weight"], "new_len": s["new_len"],
            "index": s["index"]}


def _own_attn(s):
    import paper_2608_01563_amd as mg
    c = s["case"]
    if "workspace" not in s:   # kept by the program, as for the other entry points
        need = mg.mg_attn_fwd_kv4_workspace_bytes(c["B"], c["Hq"], c["H"], c["Lq"], c["L"], c["d"],
                                                  c["weights"], c["contract"])
        s["workspace"] = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
    mg.mg_attn_fwd_kv4(s["Q"], s["cache"], s["O"], s["LSE"], s["key_len"], s["q_len"], H=c["H"],
                       L=c["L"], causal=True, scale=1.0 / math.sqrt(c["d"]), weight=s["weight"],
                       contract=c["contract"], workspace=s["workspace"])
    out = {"O": s["O"], "LSE": s["LSE"]}
    if s["weight"] is not None:
        out["weight"] = s["weight"]
    return out


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"append": _own_append, "evict": _own_evict, "attn": _own_attn}[kind](state)
    return {"append": _plain_append, "evict": _plain_evict, "attn": _plain_attn}[kind](state)


# ----------------------------------------------------------- 64-bit definitions --
def _exact_quantised(x):
    """Values of the definition for rows [n, d]; bf16 by hand, straight from 64 bits."""
    def bf16(t):   # the 45 lowest mantissa bits go, to nearest even
        bits = t.contiguous().view(torch.int64)
        return ((bits + ((1 << 44) - 1) + (bits >> 45 & 1)) >> 45 << 45).view(torch.float64)

    out = []
    for part in x.double().split(min(64, x.shape[-1]), dim=-1):
        mn = bf16(part.min(-1, keepdim=True).values)
        sc = bf16((part.max(-1, keepdim=True).values - part.min(-1, keepdim=True).values) / 15)
        code = ((part - mn) / sc).round().clamp(0, 15)
        out.append(torch.where(sc == 0, mn, sc * code + mn))
    return torch.cat(out, -1)


def _exact_rows(codes, sc, mn):
    """Values of a head's rows [n, d] from its codes and groups."""
    each = codes.shape[-1] // sc.shape[-1]
    return codes.double() * sc.double().repeat_interleave(each, -1) + \
        mn.double().repeat_interleave(each, -1)


def exact(case, seed):
    s = _inputs(case, seed)
    B, H, L, d = case["B"], case["H"], case["L"], case["d"]
    if case["kind"] == "append":
        out = {k: torch.zeros(s[k].shape, dtype=torch.float64, device="cuda") for k in ("K", "V")}
        weight = s["weight"].double()
        for b in range(B):
            n = case["n"] if s["count"] is None else int(s["count"][b])
            at = 0 if s["start"] is None else int(s["start"][b])
            weight[b, :, at:at + n] = 0
            for k in ("K", "V"):
                for h in range(H):
                    out[k][b, h, :n] = _exact_quantised(s[k][b, h, :n])
        return {**out, "weight": weight}
    if case["kind"] == "evict":
        keep = case["keep"]
        K, V = (torch.zeros(B, H, keep, d, dtype=torch.float64, device="cuda") for _ in range(2))
        weight = torch.zeros(B, H, L, dtype=torch.float64, device="cuda")
        for b in range(B):
            n = L if s["key_len"] is None else int(s["key_len"][b])
            for h in range(H):
                w = s["weight"][b, h, :n].double()
                at = torch.arange(n, device="cuda")
                if n > keep:
                    old = n - case["recent"]
                    ranked = torch.argsort(-w[:old], stable=True)[:keep - case["recent"]]
                    at = torch.cat([ranked.sort().values, at[old:]])
                K[b, h, :at.numel()] = _exact_rows(*(t[b, h][at] for t in s["k"]))
                V[b, h, :at.numel()] = _exact_rows(*(t[b, h][at] for t in s["v"]))
                weight[b, h, :at.numel()] = w[at]
        return {"K": K, "V": V, "weight": weight, "new_len": None, "index": None}
    Hq, Lq = case["Hq"], case["Lq"]
    O = torch.zeros(B, Hq, Lq, d, dtype=torch.float64, device="cuda")
    LSE = torch.full((B, Hq, Lq), -math.inf, dtype=torch.float64, device="cuda")
    weight = None if s["weight"] is None else s["weight"].double()
    for b in range(B):
        n = L if s["key_len"] is None else int(s["key_len"][b])
        rows = Lq if s["q_len"] is None else int(s["q_len"][b])
        if n == 0 or rows == 0:
            continue
        seen = torch.ones(rows, n, dtype=torch.bool, device="cuda").tril(n - rows)
        for hq in range(Hq):
            h = hq // (Hq // H)
            k, v = (_exact_rows(*(t[b, h, :n] for t in x)) for x in (s["k"], s["v"]))
            S = (s["Q"][b, hq, :rows].double() @ k.T) / math.sqrt(d)
            S = torch.where(seen, S, -math.inf)
            LSE[b, hq, :rows] = torch.logsumexp(S, 1)
            P = torch.exp(S - LSE[b, hq, :rows, None])
            P = torch.where(seen, P, 0.0)
            O[b, hq, :rows] = P @ v
            if weight is not None:
                weight[b, h, :n] += P.sum(0)
    out = {"O": O, "LSE": LSE}
    return out if weight is None else {**out, "weight": weight}


# ----------------------------------------------------------------------- work --
def work(case):
    B, H, L, d = case["B"], case["H"], case["L"], case["d"]
    row = d + 8 * _groups(d)   # bytes a token's K and V take in one head
    if case["kind"] == "append":
        e = 2 if case["contract"] == "fast_bf16" else 4
        tokens = B * H * case["n"] * (0.625 if case["ragged"] else 1)
        # rows in, cache out, weights cleared, rows out as values; about 8
        # operations a value each way
        return {"bytes": tokens * (4 * d * e + row + 4), "flops": tokens * 2 * d * 8}
    if case["kind"] == "evict":
        n = L * (0.625 if case["ragged"] else 1)
        kept = B * H * min(n, case["keep"])
        # every weight once; kept rows in and out, their weights and indices
        # out, the values read back
        return {"bytes": B * H * n * 4 + kept * (2 * row + 8 + 8 * d), "flops": kept * 4 * d}
    Hq, Lq = case["Hq"], case["Lq"]
    e = 2 if case["contract"] == "fast_bf16" else 4
    n = max(Lq, L * (0.625 if case["ragged"] else 1))
    rows = Lq * (0.75 if case["ragged"] and Lq > 1 else 1)
    pairs = B * Hq * rows * (n - (rows - 1) / 2)
    weights = 8 * B * H * n if case["weights"] else 0
    return {"bytes": B * H * n * row + 2 * B * Hq * Lq * d * e + 4 * B * Hq * Lq + weights,
            "flops": 4 * d * pairs}
