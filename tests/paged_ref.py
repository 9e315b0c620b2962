"""Plain 64-bit implementation of the paged cache (mg_paged.h) for the tests, and
bounds on what its kernels may be off by, from the roundings they make."""
import numpy as np

HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
MOST = {"bf16": float.fromhex("0x1.fep127"), "f32": float.fromhex("0x1.fffffep127")}


def pages(n, page):
    return -(-n // page)


def resize(key_len, want, table, free, count, page, T):
    """new_len, new_count, slot, offset; table and free are changed in place."""
    B, P = table.shape
    N = len(free)
    old = table.copy()
    lens = [min(max(int(n), 0), P * page) for n in key_len]
    goals = [max(int(n), 0) for n in want]
    count = min(max(int(count), 0), N)
    for b in range(B):
        for p in range(pages(goals[b], page), pages(lens[b], page)):
            if count < N:
                free[count] = old[b, p]
                count += 1
    new_len, slot, offset = [], np.full(T, -1, np.int64), [0]
    row, need_before, available = 0, 0, count
    for b in range(B):
        add = max(goals[b] - lens[b], 0)
        fits = add > 0 and goals[b] <= P * page and row + add <= T
        need = pages(goals[b], page) - pages(lens[b], page) if fits else 0
        granted = fits and (need == 0 or need_before + need <= available)
        if granted:
            for k in range(need):
                table[b, pages(lens[b], page) + k] = free[available - 1 - need_before - k]
            for j in range(add):
                pos = lens[b] + j
                e = int(table[b, pos // page])
                slot[row + j] = e * page + pos % page if 0 <= e < N else -1
            count -= need
        need_before += need
        row += add
        offset.append(min(row, T))
        new_len.append(goals[b] if add == 0 or granted else lens[b])
    return np.array(new_len), count, slot, np.array(offset)


def append(K, V, Kp, Vp, bounds, slot, kind):
    """Rows [T,H,d] into the pools [N,H,page,d] and bounds [N,H,2,d], in place."""
    N, H, page, d = Kp.shape
    runs = []   # [page, first row's place, row numbers]
    for t, s in enumerate(slot):
        if not 0 <= s < N * page:
            continue
        Kp[s // page, :, s % page], Vp[s // page, :, s % page] = K[t], V[t]
        if runs and s % page and runs[-1][3] == s - 1 and runs[-1][2][-1] == t - 1:
            runs[-1][2].append(t)
            runs[-1][3] = s
        else:
            runs.append([s // page, s % page, [t], s])
    if bounds is None:
        return
    for at, place, rows, _ in runs:
        x = K[rows].astype(np.float64)                        # [n, H, d]
        lo = np.where(np.isnan(x), MOST[kind], x).min(0)
        hi = np.where(np.isnan(x), -MOST[kind], x).max(0)
        if place:
            old = bounds[at].astype(np.float64)
            lo = np.fmin(lo, old[:, 0])
            hi = np.fmax(hi, old[:, 1])
        bounds[at, :, 0] = np.clip(lo, -MOST[kind], MOST[kind])
        bounds[at, :, 1] = np.clip(hi, -MOST[kind], MOST[kind])


def limit(n, rows, i, causal):
    """How many tokens row i sees."""
    if i >= rows:
        return 0
    return max(min(n, i + 1 + n - rows) if causal else n, 0)


def scores(q, bounds, table, m):
    """The f32 scores of the first m pages for the group's rows q [G, d]; bounds
    [N, 2, d] of the cache head."""
    N = bounds.shape[0]
    out = np.full(m, np.nan, np.float32)
    q = q.astype(np.float64)
    for p in range(m):
        if 0 <= table[p] < N:
            lo, hi = bounds[table[p]].astype(np.float64)
            with np.errstate(all="ignore"):
                each = (np.maximum(q, 0) * hi + np.minimum(q, 0) * lo).sum(1).astype(np.float32)
            if not np.isnan(each).all():
                out[p] = np.nanmax(each) + np.float32(0)
    return out


def select(q, bounds, table, m, keep, first, recent):
    """Pages kept, ascending, -1 behind the last."""
    if m <= keep:
        return list(range(m)) + [-1] * (keep - m)
    s = scores(q, bounds, table, m)
    middle = sorted(range(first, m - recent), key=lambda p: (np.isnan(s[p]), -np.float64(s[p]), p))
    return sorted(list(range(first)) + middle[:keep - first - recent] +
                  list(range(m - recent, m)))


def listed(index, table, page, n, P, N):
    """Tokens, below n, of a list's pages and where they lie (page, row)."""
    out, before = [], -1
    for k, p in enumerate(index):
        if p > before and 0 <= p < P and 0 <= table[p] < N:
            out += [(p * page + r, table[p], r) for r in range(page) if p * page + r < n]
        before = p
    return out


def attention(q, k, v, scale, kind):
    """One row's O and LSE over the tokens it sees, k, v [n, d], in 64 bits, and
    bounds on what a kernel may be off by: (O, LSE, tol_O, tol_LSE).

    Bounds.  Products of a score are exact or fused, their f32 sum is off by at
    most a half step of the sum of magnitudes each: (d + 16) of them.  p is off
    relatively by what its score and the row's sum are (twice the largest score
    error, the exponential's steps, the scores' own rounding in base 2).  In O, p
    is within 2^-15 (bf16: a part cut off, off by a step, 2^-7, and the rest rounded);
    n terms and the joins of units and waves are summed in f32; O is rounded once
    to its type."""
    n, d = k.shape
    if n == 0:
        return np.zeros(d), -np.inf, np.zeros(d), 0.0
    f32 = HALF_STEP["f32"]
    q, k, v = (x.astype(np.float64) for x in (q, k, v))
    s = scale * (k @ q)
    eS = abs(scale) * (np.abs(k) @ np.abs(q)) * (d + 16) * f32
    top = s.max()
    p = np.exp(s - top)
    LSE = top + np.log(p.sum())
    p /= p.sum()
    rel = 2 * (eS.max() + (4 + np.abs(s).max() + abs(LSE)) * 2 * f32) + (n + 16) * f32
    O = p @ v
    part = 2 * HALF_STEP["bf16"] ** 2 if kind == "bf16" else 0.0
    tO = HALF_STEP[kind] * np.abs(O) + (part + rel + (n + 16) * f32) * (p @ np.abs(v)) + 1e-37
    return O, LSE, tO, rel + 4 * f32 * abs(LSE)
