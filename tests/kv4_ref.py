"""Plain 64-bit implementation of the 4-bit cache (mg_kv4.h) for the tests, and
bounds on what its kernels may be off by, from the roundings they make."""
import numpy as np

HALF_STEP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}


def groups(d):
    return max(1, d // 64)


def bf16_round(x):
    """f32 array -> nearest bf16 (even), as f32."""
    u = np.ascontiguousarray(x, np.float32).view(np.uint32).astype(np.uint64)
    r = ((u + 0x7fff + ((u >> 16) & 1)) >> 16 << 16).astype(np.uint32).view(np.float32)
    return np.where(np.isfinite(x), r, x).astype(np.float32)


def quantise(x):
    """Codes [..., d], scale and min [..., groups] of rows x (f32 values)."""
    d = x.shape[-1]
    g = np.asarray(x, np.float32).reshape(*x.shape[:-1], groups(d), d // groups(d))
    with np.errstate(all="ignore"):
        lo, hi = g.min(-1), g.max(-1)
        mn = bf16_round(lo)
        sc = bf16_round(((hi - lo).astype(np.float32) / np.float32(15)).astype(np.float32))
        sc = np.where(sc < 2.0 ** -126, np.float32(0), sc)
        bad = ~(np.isfinite(g).all(-1) & np.isfinite(mn) & np.isfinite(sc))
        safe = np.where(sc > 0, sc, 1).astype(np.float64)
        q = (g.astype(np.float64) - mn[..., None]) / safe[..., None]
        code = np.clip(np.rint(q), 0, 15)
    code = np.where((bad | (sc == 0))[..., None], 0, code).astype(np.uint8)
    sc, mn = np.where(bad, np.nan, sc), np.where(bad, np.nan, mn)
    return code.reshape(x.shape), sc.astype(np.float32), mn.astype(np.float32)


def values(code, sc, mn):
    d = code.shape[-1]
    g = code.reshape(*code.shape[:-1], groups(d), d // groups(d)).astype(np.float64)
    return (g * sc[..., None].astype(np.float64) + mn[..., None].astype(np.float64)).reshape(
        code.shape)


def regions(B, H, L, d):
    """(byte offset, u32 shape) of the four regions, and the size."""
    Lp = (L + 31) // 32 * 32
    shapes = [(B, H, Lp, d // 8), (B, H, Lp // 8, d), (B, H, Lp, groups(d)), (B, H, Lp, groups(d))]
    out, at = [], 0
    for s in shapes:
        out.append((at, s))
        at += (int(np.prod(s)) * 4 + 255) // 256 * 256
    return out, at


class Cache:
    """A cache as codes and groups, to and from the documented bytes."""

    def __init__(self, B, H, L, d):
        self.dims = (B, H, L, d)
        Lp = (L + 31) // 32 * 32
        self.code = [np.zeros((B, H, Lp, d), np.uint8) for _ in range(2)]
        self.word = [np.zeros((B, H, Lp, groups(d)), np.uint32) for _ in range(2)]

    @classmethod
    def from_bytes(cls, raw, B, H, L, d):
        c = cls(B, H, L, d)
        parts = [raw[at:at + int(np.prod(s)) * 4].view(np.uint32).reshape(s)
                 for at, s in regions(B, H, L, d)[0]]
        ch = np.arange(d)
        kw = (ch // 8 % 4) * (d // 32) + ch // 32
        c.code[0] = (parts[0][..., kw] >> (4 * (ch % 8)).astype(np.uint32) & 15).astype(np.uint8)
        w = min(4, d // 16)
        b = ch // 16
        vw = 16 * w * (b // w) + w * (ch % 16) + b % w
        words = parts[1][..., vw]                               # [B,H,octets,d]
        t = np.arange(8, dtype=np.uint32)[:, None]
        c.code[1] = (words[..., None, :] >> (4 * t) & 15).astype(np.uint8).reshape(
            c.code[1].shape)
        c.word = [parts[2].copy(), parts[3].copy()]
        return c

    def to_bytes(self):
        B, H, L, d = self.dims
        spec, size = regions(B, H, L, d)
        raw = np.zeros(size, np.uint8)
        ch = np.arange(d)
        k = np.zeros(spec[0][1], np.uint32)
        for c in ch:
            k[..., (c // 8 % 4) * (d // 32) + c // 32] |= \
                self.code[0][..., c].astype(np.uint32) << np.uint32(4 * (c % 8))
        w = min(4, d // 16)
        v = np.zeros(spec[1][1], np.uint32)
        eight = self.code[1].reshape(*v.shape[:3], 8, d).astype(np.uint32)
        for c in ch:
            at = 16 * w * (c // 16 // w) + w * (c % 16) + c // 16 % w
            for t in range(8):
                v[..., at] |= eight[..., t, c] << np.uint32(4 * t)
        for (at, s), part in zip(spec, (k, v, *self.word)):
            b = np.ascontiguousarray(part).view(np.uint8).ravel()
            raw[at:at + b.size] = b
        return raw

    def group(self, which):
        """(scale, min) as f32."""
        w = self.word[which]
        return ((w & np.uint32(0xffff0000)).view(np.float32),
                (w << np.uint32(16)).astype(np.uint32).view(np.float32))

    def rows(self, which):
        return values(self.code[which], *self.group(which))

    def put(self, which, b, pos, x):
        """Rows x [H, m, d] of sequence b at positions pos [m]."""
        code, sc, mn = quantise(x)
        self.code[which][b][:, pos] = code
        bits = lambda f: np.where(np.isnan(f), np.uint32(0x7fc0), f.view(np.uint32) >> 16)
        self.word[which][b][:, pos] = (bits(sc) << np.uint32(16) | bits(mn)).astype(np.uint32)


def append(cache, weight, K, V, start, count):
    B, H, n, d = K.shape
    L = cache.dims[2]
    for b in range(B):
        j = np.arange(min(max(int(count[b]), 0), n))
        pos = j.astype(np.int64) + int(start[b])
        ok = (pos >= 0) & (pos < L)
        for which, x in ((0, K), (1, V)):
            cache.put(which, b, pos[ok], x[b][:, j[ok]])
        if weight is not None:
            weight[b][:, pos[ok]] = 0


def evict(weight, n, keep, recent):
    """Indices that stay of one head's n tokens."""
    if n <= keep:
        return np.arange(n)
    w = weight[:n - recent].astype(np.float64)
    w = np.where(np.isnan(w), -np.inf, w)
    nan = np.isnan(weight[:n - recent])
    order = sorted(range(n - recent), key=lambda j: (nan[j], -w[j], j))
    return np.concatenate([np.sort(np.array(order[:keep - recent], int)),
                           np.arange(n - recent, n)]).astype(int)


def attention(q, code, group, n, rows, causal, scale, strict, many=False):
    """One query head's O, LSE, P over one cache head in 64 bits, and bounds on
    what a kernel may be off by: (O, LSE, P, tol_O, tol_LSE, tol_P).

    Bounds.  A score is a sum of d products in f32 whose operands are exact
    (strict: q within 2^-23); its error is at most (d + 16) half steps of the
    sum of magnitudes.  p is off relatively by what the score is, plus the
    exponential's two ulps and the score's own rounding.  In O each p * scale
    is rounded once to f16 (strict: within 2^-23), n terms are summed in f32
    and the result is rounded to its type.  With many bf16 rows a head p and v
    are rounded to f16 each, v in units that leave an error of 2^-34 of the
    largest v at worst, and the largest p is held as 2^10 or more: p below f16's
    normal numbers are off by up to 2^-25, so by 2^-35 of the sum of p.

    Roundings are relative to the parts that a value is summed from: scale code
    and min, or, strict, scale (code - 8) and min + 8 scale (which f32 rounds
    once more: a half step of it).  p * scale is held as f16 in units of
    2^(e - 11), 2^e at most twice the largest scale: below f16's normal numbers it
    is off by up to 2^-25 units, times a code of 15 (strict: 8) for each token."""
    Lq, d = q.shape
    (kc, vc), ((ks, km), (vs, vm)) = code, group
    f32 = HALF_STEP["f32"]
    k, v = values(kc[:n], ks[:n], km[:n]), values(vc[:n], vs[:n], vm[:n])
    def size(c, s, m):
        if not strict:
            return values(c, np.abs(s), np.abs(m))
        return values(np.abs(c.astype(np.int16) - 8), np.abs(s), np.abs(m + 8 * s))

    kk, vv = size(kc[:n], ks[:n], km[:n]), size(vc[:n], vs[:n], vm[:n])
    i = np.arange(Lq)[:, None]
    j = np.arange(n)[None, :]
    seen = (i < rows) & (~np.bool_(causal) | (j <= i + n - rows)) if causal else \
        np.broadcast_to(i < rows, (Lq, n))
    S = scale * (q @ k.T)
    eS = abs(scale) * (np.abs(q) @ kk.T) * (d + 16 + (4 if strict else 0)) * f32
    O, LSE = np.zeros((Lq, d)), np.full(Lq, -np.inf)
    P = np.zeros((Lq, n))
    tO, tL, tP = np.zeros((Lq, d)), np.zeros(Lq), np.zeros((Lq, n))
    for r in range(Lq):
        at = np.nonzero(seen[r])[0]
        if not len(at):
            continue
        s = S[r, at]
        top = s.max()
        p = np.exp(s - top)
        LSE[r] = top + np.log(p.sum())
        p /= p.sum()
        rel = 2 * (eS[r, at].max() + (4 + np.abs(s).max() + abs(LSE[r])) * 2 * f32) \
            + len(at) * f32
        P[r, at] = p
        O[r] = p @ v[at]
        out = f32 if strict else HALF_STEP["bf16"]
        part = 2.0 ** -22 if strict else HALF_STEP["f16"] * (2 if many else 1)
        tO[r] = out * np.abs(O[r]) + (part + rel + (len(at) + 8) * f32) * (p @ vv[at]) \
            + ((2.0 ** -34 + len(at) * 2.0 ** -35) * vv.max() if many else
               len(at) * (8 if strict else 15) * 2.0 ** -35 * vs[at].max())
        tL[r] = rel + 4 * f32 * abs(LSE[r])
        tP[r, at] = 2 * rel * p + 1e-30
    return O, LSE, P, tO, tL, tP
