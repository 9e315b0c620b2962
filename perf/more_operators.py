"""The operators of the paged key/value cache whose speed counts for a user of
this library, each in its plain form (elementary torch operations in 32 bits)
and through the library's entry points.

K and V live in pools of N pages, [N, H, page, d]; a sequence's token j is row
j % page of page table[b][j // page].  A case is one pass: sequences brought to
new lengths, with the pages they take and give back and the slots their new
tokens get (`mg_paged_resize`); rows written through the slots, with the
smallest and largest K of every page and channel kept (`mg_paged_append`);
attention of one or a few new tokens over the pages (`mg_attn_fwd_paged`); or
the same over the pages only whose bounds promise the largest scores
(`mg_paged_select`, `mg_attn_fwd_paged_sparse`).
"""
import math

import torch

own = False

_MAX = {torch.bfloat16: 3.3895313892515355e38, torch.float32: 3.4028234663852886e38}


# ---------------------------------------------------------------------- cases --
def _resize(name, B, P, page, T, want, short):
    """B sequences with room for P pages each.  want "tokens": one more token
    each, but for those that end or lose drafted tokens; "prompts": most are
    empty and get a prompt, T rows in all at most; short: the free pages do not
    suffice."""
    return {"name": name, "kind": "resize", "B": B, "P": P, "page": page, "T": T, "want": want,
            "short": short}


def _append(name, B, H, n, T, page, d, contract, ragged):
    """n new tokens a sequence at most, T rows at most in all (those behind the
    last have no slot); ragged: every sequence has its own length and its own
    number of new tokens."""
    return {"name": name, "kind": "append", "B": B, "H": H, "n": n, "T": T, "page": page, "d": d,
            "contract": contract, "ragged": ragged}


def _attn(name, B, Hq, H, Lq, n, room, page, d, contract, ragged, empty=False):
    """Lq query rows (a sequence's last tokens, causal) of Hq heads over H cache
    heads of up to n tokens, in tables with room for `room` tokens; ragged:
    sequences of a quarter and more, and for Lq > 1 some with fewer rows; empty:
    the first sequence holds nothing."""
    return {"name": name, "kind": "attn", "B": B, "Hq": Hq, "H": H, "Lq": Lq, "n": n, "room": room,
            "page": page, "d": d, "contract": contract, "ragged": ragged, "empty": empty}


def _sparse(name, B, Hq, H, Lq, n, page, d, keep, contract, ragged):
    """As _attn, over `keep` pages a row and cache head: the first, the last two
    and those whose bounds promise the largest scores."""
    return {"name": name, "kind": "sparse", "B": B, "Hq": Hq, "H": H, "Lq": Lq, "n": n, "room": n,
            "page": page, "d": d, "keep": keep, "contract": contract, "ragged": ragged,
            "empty": False}


def listed():
    return [
        # the step of a served batch: a token more a sequence, some end, some are cut back
        _resize("resize tokens", 256, 512, 16, 256, "tokens", False),
        # prompts of a batch come in, more of them than the pool has pages for
        _resize("resize prompts short", 64, 256, 64, 200000, "prompts", True),
        # a decode step's rows: one token a sequence
        _append("append tokens bf16", 64, 8, 1, 64, 64, 128, "fast_bf16", True),
        # the packed rows of a batch of prompts
        _append("append prompts bf16", 8, 8, 4096, 8 * 4096, 16, 128, "fast_bf16", True),
        # odd lengths in full precision, six heads of 64, going on inside a page
        _append("append ragged f32", 3, 6, 500, 1500, 32, 64, "strict_f32", True),
        # the smallest decode step: launches and latency
        _attn("decode tiny bf16", 1, 4, 4, 1, 256, 256, 16, 64, "fast_bf16", False),
        # an ordinary served batch: grouped heads, small pages, tables with room to grow
        _attn("decode grouped bf16", 32, 32, 8, 1, 4096, 16384, 16, 128, "fast_bf16", True, True),
        # a long-context batch, the largest cache
        _attn("decode long bf16", 8, 32, 8, 1, 65536, 65536, 64, 128, "fast_bf16", True),
        # full-precision queries, a head of its own each, odd length
        _attn("decode ragged f32", 2, 6, 6, 1, 1500, 2048, 32, 64, "strict_f32", True),
        # seven drafted tokens a sequence scored at once
        _attn("draft rows bf16", 8, 32, 8, 7, 4001, 8192, 64, 128, "fast_bf16", True),
        # the long-context batch again, an eighth and less of it read
        _sparse("sparse long bf16", 8, 32, 8, 1, 65536, 64, 128, 64, "fast_bf16", True),
        # a few sequences in full precision
        _sparse("sparse ragged f32", 3, 6, 6, 1, 9001, 32, 64, 24, "strict_f32", True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    what = rng.random()
    d = rng.choice((32, 64, 128, 128))
    contract = rng.choice(("fast_bf16", "fast_bf16", "strict_f32"))
    page = rng.choice((16, 32, 64, 128))
    H = rng.choice((1, 2, 4, 6, 8))
    if what < 0.2:
        want = rng.choice(("tokens", "prompts"))
        B, P = _log(rng, 1, 1024), max(1, _log(rng, 64, 16384) // page)
        T = B if want == "tokens" else min(200000, max(B, int(B * P * page * rng.uniform(0.3, 1))))
        while B * P > 200000:
            B, T = B // 2, max(1, T // 2)
        c = _resize("", B, P, page, T, want, rng.random() < 0.4)
    elif what < 0.4:
        B, n = _log(rng, 1, 64), rng.choice((1, _log(rng, 1, 4096)))
        while B * n * H * d > 3e7 or B * max(n, page) * H * d > 5e7:
            B, n = max(1, B // 2), max(1, n - n // 8)
        c = _append("", B, H, n, B * n, page, d, contract, rng.random() < 0.7)
    elif what < 0.75:
        Lq = rng.choice((1, 1, 1, rng.randint(2, 9)))
        n, B = max(Lq, _log(rng, 16, 65536)), _log(rng, 1, 48)
        G = rng.choice((1, 2, 4, 8, 16))
        while B > 1 and (B * H * n * d > 2.6e8 or B * H * G * Lq * n > 1.5e8):
            B = B // 2
        while G > 1 and B * H * G * Lq * n > 1.5e8:
            G = G // 2
        c = _attn("", B, H * G, H, Lq, n, n * rng.choice((1, 1, 2, 5)), page, d, contract,
                  rng.random() < 0.7, rng.random() < 0.1)
    else:
        Lq = rng.choice((1, 1, 1, rng.randint(2, 5)))
        n, B, G = max(Lq, _log(rng, 64, 65536)), _log(rng, 1, 16), rng.choice((1, 2, 4, 8))
        while B > 1 and B * H * n * d > 2.6e8:
            B = B // 2
        keep = max(4, int(-(-n // page) * rng.uniform(0.02, 0.7)))
        while keep > 8 and B * H * G * Lq * keep * page * d > 2e9:
            keep = keep // 2
        c = _sparse("", B, H * G, H, Lq, n, page, d, keep, contract, rng.random() < 0.7)
    return {k: v for k, v in c.items() if k != "name"}


# ---------------------------------------------------------------------- inputs --
def _pages(n, page):
    return -(-n // page)


def _dtype(c):
    return torch.bfloat16 if c["contract"] == "fast_bf16" else torch.float32


def _ints(g, lo, hi, B):
    return torch.randint(lo, max(hi, lo) + 1, (B,), generator=g, device="cuda")


def _pool(g, N, H, page, d, dtype, topic=None):
    """Rows as a model leaves them: channels of different size, some off zero."""
    size = torch.exp(0.5 * torch.randn(H, 1, d, generator=g, device="cuda"))
    off = torch.randn(H, 1, d, generator=g, device="cuda") * 0.5
    out = torch.empty(N, H, page, d, dtype=dtype, device="cuda")
    step = max(1, (1 << 27) // (H * page * d))
    for i in range(0, N, step):
        x = torch.randn(out[i:i + step].shape, generator=g, device="cuda") * size + off
        out[i:i + step] = x if topic is None else x + topic[i:i + step]
    return out


def _resize_inputs(c, g):
    B, P, page, N = c["B"], c["P"], c["page"], c["B"] * c["P"]
    s = {"case": c}
    if c["want"] == "tokens":
        length = _ints(g, 0, P * page - 1, B)
        want = length + 1
        u = torch.rand(B, generator=g, device="cuda")
        want = torch.where(u < 0.05, 0, torch.where(u < 0.1, (length - 3).clamp(min=0), want))
    else:
        u = torch.rand(B, generator=g, device="cuda")
        length = torch.where(u < 0.2, _ints(g, 0, P * page // 2, B), 0)
        want = length + _ints(g, 1, max(1, 2 * c["T"] // B), B)   # about T rows, or more
        want = torch.where(u < 0.1, 0, want.clamp(max=P * page))
    # pages in an order that many requests have left behind
    order = torch.randperm(N, generator=g, device="cuda").view(B, P)
    held = torch.arange(P, device="cuda") < _pages(length, page)[:, None]
    s["free"] = order.flatten()[torch.argsort(held.flatten().int(), stable=True)].int()
    left = (~held).sum()
    need = (_pages(want, page) - _pages(length, page)).clamp(min=0).sum()
    if c["short"]:
        left = torch.minimum(left, need * 2 // 3)
    s["free_count"] = left.reshape(1).int()
    s["table"] = torch.where(held, order, -1).int()
    s["key_len"], s["want"] = length.int(), want.int()
    return s


def _append_inputs(c, g):
    B, H, n, T, page, d = (c[k] for k in ("B", "H", "n", "T", "page", "d"))
    s = {"case": c}
    start = _ints(g, 0, 2 * page, B) if c["ragged"] else torch.zeros(B, dtype=torch.int64,
                                                                    device="cuda")
    count = _ints(g, max(1, n // 4), n, B) if c["ragged"] else torch.full((B,), n, device="cuda")
    P = _pages(2 * page + n, page)
    N = B * P
    table = torch.randperm(N, generator=g, device="cuda").view(B, P)
    end = count.cumsum(0)
    t = torch.arange(T, device="cuda")
    b = torch.searchsorted(end, t, right=True).clamp(max=B - 1)
    pos = (start[b] + t - (end - count)[b]).clamp(max=P * page - 1)
    slot = table[b, pos // page] * page + pos % page
    s["slot"] = torch.where(t < end[-1], slot, -1).int()
    s["table"], s["start"], s["count"] = table, start, count
    s["K"], s["V"] = (torch.randn(T, H, d, generator=g, device="cuda").to(_dtype(c))
                      for _ in range(2))
    s["Kp"], s["Vp"] = (_pool(g, N, H, page, d, _dtype(c)) for _ in range(2))
    s["bounds"] = _bounds_of(s["Kp"])
    return s


def _bounds_of(Kp):
    return torch.stack([Kp.amin(2), Kp.amax(2)], dim=2)


def _attn_inputs(c, g):
    B, Hq, H, Lq, n, page, d = (c[k] for k in ("B", "Hq", "H", "Lq", "n", "page", "d"))
    s = {"case": c}
    most, P = _pages(n, page), _pages(c["room"], page)
    N = B * most + 3
    order = torch.randperm(N, generator=g, device="cuda")[:B * most].view(B, most)
    s["table"] = torch.nn.functional.pad(order, (0, P - most), value=-1).int().contiguous()
    lens = _ints(g, max(Lq, n // 4), n, B) if c["ragged"] else torch.full((B,), n, device="cuda")
    s["q_len"] = _ints(g, max(1, Lq // 2), Lq, B).int() if c["ragged"] and Lq > 1 else None
    if c["empty"]:
        lens[0] = 0
        if s["q_len"] is not None:
            s["q_len"][0] = 0
    s["key_len"] = lens.int()
    topic = None
    Q = torch.randn(B, Hq, Lq, d, generator=g, device="cuda")
    if c["kind"] == "sparse":
        # what neighbouring tokens share, and queries that look for some of it
        topic = torch.randn(N, H, 1, d, generator=g, device="cuda")
        at = order[torch.arange(B, device="cuda")[:, None],
                   _ints(g, 0, most - 1, B * Lq).view(B, Lq)]
        seek = topic[at, :, 0].permute(0, 2, 1, 3)
        Q = Q + 0.5 * seek.repeat_interleave(Hq // H, 1)
    s["Q"] = Q.to(_dtype(c))
    s["Kp"] = _pool(g, N, H, page, d, _dtype(c), topic)
    s["Vp"] = _pool(g, N, H, page, d, _dtype(c))
    if c["kind"] == "sparse":
        s["bounds"] = _bounds_of(s["Kp"])
    return s


def _inputs(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return {"resize": _resize_inputs, "append": _append_inputs, "attn": _attn_inputs,
            "sparse": _attn_inputs}[c["kind"]](c, g)


def prepare(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "resize":
        def ints(n):
            return torch.zeros(n, dtype=torch.int32, device="cuda")

        s["new_len"], s["new_count"] = ints(case["B"]), ints(1)
        s["slot"], s["offset"] = ints(case["T"]), ints(case["B"] + 1)
    if case["kind"] in ("attn", "sparse"):
        s["O"] = torch.empty_like(s["Q"])
        s["LSE"] = torch.empty(s["Q"].shape[:3], device="cuda")
    if case["kind"] == "sparse":
        s["index"] = torch.zeros(case["B"], case["H"], case["Lq"], case["keep"],
                                 dtype=torch.int32, device="cuda")
    return s


# ---------------------------------------------------------------- plain forms --
def _plain_resize(s):
    c = s["case"]
    B, P, page, T = c["B"], c["P"], c["page"], c["T"]
    N = s["free"].numel()
    length = s["key_len"].to(torch.int64).clamp(0, P * page)
    goal = s["want"].to(torch.int64).clamp(min=0)
    have, then = _pages(length, page), _pages(goal, page)
    p = torch.arange(P, device="cuda")
    # pages given back go on the stack, a sequence after the other
    back = (have - then).clamp(min=0)
    count = s["free_count"].to(torch.int64).clamp(0, N)
    leaves = (p >= then[:, None]) & (p < have[:, None])
    to = count + (back.cumsum(0) - back)[:, None] + p - then[:, None]
    free = torch.nn.functional.pad(s["free"], (0, 1))
    free[torch.where(leaves, to, N).clamp(max=N)] = s["table"]
    free = free[:N]
    count = (count + back.sum()).clamp(max=N)
    # growing sequences take from its top while it lasts
    add = (goal - length).clamp(min=0)
    end = add.cumsum(0)
    fits = (add > 0) & (goal <= P * page) & (end <= T)
    need = torch.where(fits, then - have, 0)
    taken = need.cumsum(0)
    granted = fits & ((need == 0) | (taken <= count))
    comes = granted[:, None] & (p >= have[:, None]) & (p < then[:, None])
    at = count - 1 - ((taken - need)[:, None] + p - have[:, None])
    table = torch.where(comes, free[at.clamp(0, N - 1)], s["table"])
    t = torch.arange(T, device="cuda")
    b = torch.searchsorted(end, t, right=True).clamp(max=B - 1)
    pos = length[b] + t - (end - add)[b]
    slot = table[b, (pos // page).clamp(0, P - 1)] * page + pos % page
    slot = torch.where((t < end[-1]) & granted[b], slot, -1)
    return {"new_len": torch.where((add == 0) | granted, goal, length).int(),
            "new_count": (count - torch.where(granted, need, 0).sum()).int(), "free": free,
            "table": table, "slot": slot.int(),
            "offset": torch.nn.functional.pad(end, (1, 0)).clamp(max=T).int()}


def _plain_append(s):
    c = s["case"]
    page = c["page"]
    N, H, _, d = s["Kp"].shape
    slot = s["slot"].to(torch.int64)
    there = slot >= 0
    # a row without a slot repeats the first one that has one
    row = torch.where(there, torch.arange(slot.numel(), device="cuda"), there.int().argmax())
    slot = slot[row]
    at, off = slot // page, slot % page
    K, V = s["K"][row], s["V"][row]
    s["Kp"][at, :, off], s["Vp"][at, :, off] = K, V
    # pages that begin anew forget what they held
    begun = torch.zeros(N, dtype=torch.int32, device="cuda")
    begun.index_reduce_(0, at, (off == 0).int(), "amax")
    most = _MAX[s["Kp"].dtype]
    lo, hi = (torch.where(begun.bool()[:, None, None], e, s["bounds"][:, :, i].float())
              .reshape(N, H * d) for i, e in ((0, most), (1, -most)))
    x = K.float().reshape(-1, H * d)
    lo.index_reduce_(0, at, x, "amin")
    hi.index_reduce_(0, at, x, "amax")
    s["bounds"].copy_(torch.stack([lo.view(N, H, d), hi.view(N, H, d)], dim=2))
    return {"Kp": s["Kp"], "Vp": s["Vp"], "bounds": s["bounds"]}


def _limits(s):
    """How many tokens each row sees, [B, Lq]."""
    c = s["case"]
    n = s["key_len"].to(torch.int64)[:, None]
    rows = torch.full_like(n, c["Lq"]) if s["q_len"] is None else \
        s["q_len"].to(torch.int64)[:, None]
    i = torch.arange(c["Lq"], device="cuda")
    return torch.where(i < rows, (i + 1 + n - rows).clamp(min=0), 0)


def _plain_softmax(S, V, dtype):
    """O and LSE of scores S [.., rows, tokens] and values V [.., tokens, d]."""
    top = S.amax(-1, keepdim=True)
    P = torch.exp(S - torch.where(top == -math.inf, 0.0, top))
    sums = P.sum(-1, keepdim=True)
    O = torch.matmul(P / torch.where(sums > 0, sums, 1.0), V)
    LSE = torch.where(sums > 0, top + torch.log(sums), -math.inf).squeeze(-1)
    return O.to(dtype), LSE


def _plain_attn(s):
    c = s["case"]
    B, Hq, H, Lq, n, page, d = (c[k] for k in ("B", "Hq", "H", "Lq", "n", "page", "d"))
    table = s["table"][:, :_pages(n, page)].clamp(min=0).to(torch.int64)
    K, V = (x[table].transpose(1, 2).float().reshape(B, H, -1, d) for x in (s["Kp"], s["Vp"]))
    Q = s["Q"].float().reshape(B, H, Hq // H * Lq, d)
    S = torch.matmul(Q, K.transpose(2, 3).contiguous()).reshape(B, H, Hq // H, Lq, -1)
    seen = torch.arange(K.shape[2], device="cuda") < _limits(s)[:, None, None, :, None]
    S = (S / math.sqrt(d)).masked_fill(~seen, -math.inf).reshape(B, H, Hq // H * Lq, -1)
    O, LSE = _plain_softmax(S, V, s["Q"].dtype)
    return {"O": O.reshape(B, Hq, Lq, d), "LSE": LSE.reshape(B, Hq, Lq)}


def _plain_select(s):
    """Pages [B, H, Lq, keep], ascending, -1 behind the last."""
    c = s["case"]
    B, Hq, H, Lq, n, page, d, keep = (c[k] for k in
                                      ("B", "Hq", "H", "Lq", "n", "page", "d", "keep"))
    table = s["table"].clamp(min=0).to(torch.int64)
    # in 64 bits: pages next to the border of what is kept must fall on their own side
    lo, hi = (s["bounds"][:, :, i][table].permute(0, 2, 3, 1).double().contiguous()
              for i in range(2))
    Q = s["Q"].double().reshape(B, H, Hq // H * Lq, d)
    score = (torch.matmul(Q.clamp(min=0), hi) + torch.matmul(Q.clamp(max=0), lo)) \
        .reshape(B, H, Hq // H, Lq, -1).amax(2).float()
    left = _pages(_limits(s), page)[:, None, :, None]      # pages a row sees
    p = torch.arange(score.shape[-1], device="cuda")
    score = score.masked_fill((p < 1) | (p >= left - 2), math.inf).masked_fill(p >= left, -math.inf)
    # the stable order puts equal scores by their index
    best = torch.sort(score, dim=3, descending=True, stable=True).indices[..., :keep]
    best = torch.nn.functional.pad(best, (0, keep - best.shape[-1]), value=score.shape[-1])
    gone = torch.arange(keep, device="cuda") >= left
    best = torch.sort(best.masked_fill(gone, score.shape[-1]), dim=3).values
    return best.masked_fill(gone, -1).int()


def _plain_sparse(s):
    c = s["case"]
    B, Hq, H, Lq, page, d, keep = (c[k] for k in ("B", "Hq", "H", "Lq", "page", "d", "keep"))
    G = Hq // H
    index = _plain_select(s)
    b, h = torch.arange(B, device="cuda"), torch.arange(H, device="cuda")
    p = index.clamp(min=0).to(torch.int64)
    at = s["table"].clamp(min=0).to(torch.int64)[b[:, None, None, None], p]
    K, V = (x[at, h[:, None, None]].float().reshape(B * H * Lq, keep * page, d)
            for x in (s["Kp"], s["Vp"]))
    Q = s["Q"].float().reshape(B, H, G, Lq, d).transpose(2, 3).reshape(B * H * Lq, G, d)
    S = torch.matmul(Q, K.transpose(1, 2).contiguous()) / math.sqrt(d)
    token = p[..., None] * page + torch.arange(page, device="cuda")
    seen = (index >= 0)[..., None] & (token < _limits(s)[:, None, :, None, None])
    S = S.masked_fill(~seen.reshape(B * H * Lq, 1, -1), -math.inf)
    O, LSE = _plain_softmax(S, V, s["Q"].dtype)
    return {"index": index,
            "O": O.view(B, H, Lq, G, d).transpose(2, 3).reshape(B, Hq, Lq, d),
            "LSE": LSE.view(B, H, Lq, G).transpose(2, 3).reshape(B, Hq, Lq)}


# ------------------------------------------------------- the library's entry points --
def _workspace(s, name, need):
    """Kept by the program, as for the other entry points."""
    if name not in s:
        s[name] = torch.empty(max(need(), 1), dtype=torch.uint8, device="cuda")
    return s[name]


def _own_resize(s):
    import paper_2608_01563_amd as mg
    c = s["case"]
    ws = _workspace(s, "ws", lambda: mg.mg_paged_resize_workspace_bytes(c["B"], c["T"]))
    mg.mg_paged_resize(s["key_len"], s["want"], s["table"], s["free"], s["free_count"],
                       s["new_len"], s["new_count"], s["slot"], s["offset"], page=c["page"],
                       workspace=ws)
    return {k: s[k] for k in ("new_len", "new_count", "free", "table", "slot", "offset")}


def _own_append(s):
    import paper_2608_01563_amd as mg
    mg.mg_paged_append(s["K"], s["V"], s["Kp"], s["Vp"], s["slot"], s["bounds"],
                       contract=s["case"]["contract"])
    return {k: s[k] for k in ("Kp", "Vp", "bounds")}


def _own_attn(s):
    import paper_2608_01563_amd as mg
    c = s["case"]
    ws = _workspace(s, "ws", lambda: mg.mg_attn_fwd_paged_workspace_bytes(
        c["B"], c["Hq"], c["H"], c["Lq"], c["d"], c["page"], s["table"].shape[1], c["contract"]))
    mg.mg_attn_fwd_paged(s["Q"], s["Kp"], s["Vp"], s["table"], s["key_len"], s["O"], s["LSE"],
                         s["q_len"], causal=True, scale=1.0 / math.sqrt(c["d"]),
                         contract=c["contract"], workspace=ws)
    return {"O": s["O"], "LSE": s["LSE"]}


def _own_sparse(s):
    import paper_2608_01563_amd as mg
    c = s["case"]
    wsel = _workspace(s, "wsel", lambda: mg.mg_paged_select_workspace_bytes(
        c["B"], c["Hq"], c["H"], c["Lq"], c["d"], c["page"], s["table"].shape[1], c["contract"]))
    mg.mg_paged_select(s["Q"], s["bounds"], s["table"], s["key_len"], s["index"], s["q_len"],
                       page=c["page"], causal=True, first=1, recent=2, contract=c["contract"],
                       workspace=wsel)
    ws = _workspace(s, "ws", lambda: mg.mg_attn_fwd_paged_sparse_workspace_bytes(
        c["B"], c["Hq"], c["H"], c["Lq"], c["d"], c["page"], c["keep"], c["contract"]))
    mg.mg_attn_fwd_paged_sparse(s["Q"], s["Kp"], s["Vp"], s["table"], s["key_len"], s["index"],
                                s["O"], s["LSE"], s["q_len"], causal=True,
                                scale=1.0 / math.sqrt(c["d"]), contract=c["contract"],
                                workspace=ws)
    return {"index": s["index"], "O": s["O"], "LSE": s["LSE"]}


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"resize": _own_resize, "append": _own_append, "attn": _own_attn,
                "sparse": _own_sparse}[kind](state)
    return {"resize": _plain_resize, "append": _plain_append, "attn": _plain_attn,
            "sparse": _plain_sparse}[kind](state)


# ----------------------------------------------------------- 64-bit definitions --
def _exact_append(s):
    c = s["case"]
    page = c["page"]
    out = {k: s[k].double() for k in ("Kp", "Vp", "bounds")}
    t = 0
    for b, (at, n) in enumerate(zip(s["start"].tolist(), s["count"].tolist())):
        while n > 0:   # a page at a time
            row, m = int(s["table"][b, at // page]), min(n, page - at % page)
            new = s["K"][t:t + m].double().transpose(0, 1)
            out["Kp"][row, :, at % page:at % page + m] = new
            out["Vp"][row, :, at % page:at % page + m] = s["V"][t:t + m].double().transpose(0, 1)
            lo, hi = new.min(1).values, new.max(1).values
            if at % page:
                lo = torch.minimum(lo, out["bounds"][row, :, 0])
                hi = torch.maximum(hi, out["bounds"][row, :, 1])
            out["bounds"][row, :, 0], out["bounds"][row, :, 1] = lo, hi
            t, at, n = t + m, at + m, n - m
    return out


def _exact_pages(s, b, h, q, n):
    """The pages of one row and cache head: q its group's rows [G, d], n tokens seen."""
    c = s["case"]
    m = -(-n // c["page"])
    if m <= c["keep"]:
        return list(range(m))
    bound = s["bounds"][s["table"][b, :m].long(), h].double()
    score = torch.stack([torch.where(r > 0, r * bound[:, 1], r * bound[:, 0]).sum(1) for r in q])
    score = score.max(0).values.float().tolist()
    fixed = [0] + list(range(m - 2, m))
    others = sorted(range(1, m - 2), key=lambda j: (-score[j], j))
    return sorted(fixed + others[:c["keep"] - 3])


def _exact_attn(s):
    c = s["case"]
    B, Hq, H, Lq, page, d = (c[k] for k in ("B", "Hq", "H", "Lq", "page", "d"))
    G = Hq // H
    O = torch.zeros(B, Hq, Lq, d, dtype=torch.float64, device="cuda")
    LSE = torch.full((B, Hq, Lq), -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(s["key_len"].tolist()):
        rows = Lq if s["q_len"] is None else int(s["q_len"][b])
        held = s["table"][b, :-(-n // page)].long()
        for h in range(H if n else 0):
            k, v = (x[held, h].double().reshape(-1, d) for x in (s["Kp"], s["Vp"]))
            for i in range(rows):
                q, sees = s["Q"][b, h * G:(h + 1) * G, i].double(), i + 1 + n - rows
                if sees <= 0:
                    continue
                if c["kind"] == "sparse":
                    at = torch.tensor(_exact_pages(s, b, h, q, sees), device="cuda")
                    at = (at[:, None] * page + torch.arange(page, device="cuda")).flatten()
                    at = at[at < sees]
                    ki, vi = k[at], v[at]
                else:
                    ki, vi = k[:sees], v[:sees]
                S = (ki @ q.T).T / math.sqrt(d)
                z = torch.logsumexp(S, 1)
                LSE[b, h * G:(h + 1) * G, i] = z
                O[b, h * G:(h + 1) * G, i] = torch.exp(S - z[:, None]) @ vi
    return {"O": O, "LSE": LSE}


def exact(case, seed):
    if case["kind"] == "resize":   # whole numbers only
        return None
    s = _inputs(case, seed)
    if case["kind"] == "append":
        return _exact_append(s)
    if case["kind"] == "attn":
        return _exact_attn(s)
    return {"index": None, **_exact_attn(s)}


# ----------------------------------------------------------------------- work --
def work(case):
    c = case
    B, page = c["B"], c["page"]
    if c["kind"] == "resize":
        # lengths in and out, offsets, slots; the pages that change hands, read
        # and written; a few operations a slot
        pages = B / page if c["want"] == "tokens" else c["T"] / page
        return {"bytes": 4 * (4 * B + c["T"] + 4 * pages), "flops": 4 * c["T"]}
    H, d = c["H"], c["d"]
    e = 2 if c["contract"] == "fast_bf16" else 4
    if c["kind"] == "append":
        n = c["n"] * (0.625 if c["ragged"] and c["n"] > 1 else 1)
        # rows in and out, slots, bounds out (and in, of the pages gone on with)
        pages = B * (n / page + 1)
        return {"bytes": B * n * (4 * H * d * e + 4) + (pages + B) * 2 * H * d * e,
                "flops": B * n * H * d * 2}
    Hq, Lq = c["Hq"], c["Lq"]
    n = max(Lq, c["n"] * (0.625 if c["ragged"] else 1))
    rows = Lq * (0.75 if c["ragged"] and Lq > 1 else 1)
    around = 2 * B * Hq * Lq * d * e + 4 * B * Hq * Lq
    if c["kind"] == "attn":
        return {"bytes": B * H * n * 2 * d * e + 4 * B * n / page + around,
                "flops": 4 * d * B * Hq * rows * (n - (rows - 1) / 2)}
    kept = min(n, c["keep"] * page)
    # bounds once, the listed pages of every row and head once
    return {"bytes": B * H * n / page * 2 * d * e + B * H * rows * kept * 2 * d * e +
            4 * B * H * Lq * c["keep"] + around,
            "flops": B * Hq * rows * (4 * d * kept + 4 * d * n / page)}
