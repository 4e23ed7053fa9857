"""Plain forms of the generator's operators in 64 bits (helper, not a test module): written from the definitions in
``include/ralm.h``, request by request and token by token, on numpy arrays."""
import math

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def four_bits(x):
    """The numbers that x [..., d] stands for in the cache's format."""
    x = np.asarray(x, dtype=np.float64)
    b = x.reshape(x.shape[:-1] + (-1, 32))
    out = np.empty_like(b)
    for at in np.ndindex(b.shape[:-1]):
        row = b[at]
        if not np.isfinite(row).all():
            out[at] = np.nan
            continue
        top = np.abs(row).max()
        e = -126
        if top > 0:
            e = max(-126, math.frexp(top)[1] - 4)
            while top > 6.0 * 2.0 ** e:
                e += 1
        e = min(e, 125)
        y = np.abs(row) / 2.0 ** e
        far = np.abs(y[:, None] - GRID)
        near = far.argmin(1)                                       # the lower one on ties ...
        up = np.minimum(near + 1, 7)
        tie = (far[np.arange(32), up] == far[np.arange(32), near]) & (near % 2 == 1)
        near = np.where(tie, up, near)                             # ... unless its code is odd
        out[at] = np.copysign(GRID[near] * 2.0 ** e, row)
    return out.reshape(x.shape)


def attention(q, K, V, scale, window=0, sinks=0):
    """q [s, Hq, d]: the last s of the n tokens of K, V [n, Hkv, d].  (out, lse, sum of the weights' |V|, (largest sum of a
    score's magnitudes per row, sum of |V|))."""
    s, Hq, d = q.shape
    n, Hkv = K.shape[:2]
    G = Hq // Hkv
    out, mag = np.zeros((s, Hq, d)), np.zeros((s, Hq, d))
    lse, size, total = np.full((s, Hq), -np.inf), np.zeros((s, Hq)), np.zeros((s, Hq, d))
    for i in range(s):
        p = n - s + i
        j = np.arange(n)
        sees = j <= p
        if window > 0:
            sees &= (j > p - window) | (j < sinks)
        j = j[sees]
        if len(j) == 0:
            continue
        for h in range(Hq):
            k, v = K[j, h // G], V[j, h // G]
            x = (k @ q[i, h]) * scale
            top = x.max()
            w = np.exp(x - top)
            out[i, h] = (w @ v) / w.sum()
            mag[i, h] = (w @ np.abs(v)) / w.sum()
            total[i, h] = np.abs(v).sum(0)
            lse[i, h] = top + math.log(w.sum())
            size[i, h] = (np.abs(k) @ np.abs(q[i, h])).max() * scale
    return out, lse, mag, (size, total)


def attention_tolerance(dtype, out, mag, size, d):
    """Per element.  Rounding to bf16 (8 significant bits) moves a number by at most 2^-8 of it, to fp16 (11 bits) by 2^-11, at least
    2^-25.  A weight's rounding is that of bf16 (fp16 queries: two bf16 numbers, 2^-16), the output's that of its type; a score's d fp32
    additions and its factor are (d + 4) 2^-24 of the sum of its magnitudes, twice that for the weight's share of the sum; an exponential, a
    sum and a quotient together are 2^-20 of the result.  Weights below 2^-126, fp32's smallest normal number, may vanish."""
    size, total = size
    w, o, least = (2.0 ** -8, 2.0 ** -8, 0.0) if dtype == "bf16" else (2.0 ** -16, 2.0 ** -11, 2.0 ** -25)
    score = 2.0 * (d + 4) * 2.0 ** -24 * size[..., None]
    return o * np.abs(out) * 1.01 + least + 2.0 ** -126 * total + (w + 2.0 ** -20 + score) * mag * 1.01


def reserve(table, lens, refs, grow, T):
    """(table, lens, refs, granted, copies) behind a reservation, from the definition."""
    table, lens, refs = table.copy(), lens.copy(), refs.copy()
    before = refs.copy()
    free = list(np.nonzero(before == 0)[0])
    granted, copies, wanted = np.zeros(len(lens), np.int32), [], 0
    for r, more in enumerate(grow):
        more = max(int(more), 0)
        have, want = -(-int(lens[r]) // T), -(-(int(lens[r]) + more) // T)
        if more == 0:
            granted[r] = 1
            continue
        if lens[r] + more > table.shape[1] * T:
            continue
        shared = lens[r] % T != 0 and before[table[r, have - 1]] > 1
        need = want - have + int(shared)
        first = wanted
        wanted += need
        if need and wanted > len(free):
            continue
        granted[r] = 1
        new = free[first:first + need]
        at = have
        if shared:
            old = table[r, have - 1]
            copies.append((int(old), int(new[0])))
            refs[old] -= 1
            at = have - 1
        for page in new:
            table[r, at] = page
            refs[page] = 1
            at += 1
        lens[r] += more
    return table, lens, refs, granted, copies


def verify_draft(ids, target, u, u_next, off, draft=None):
    """(accepted, next) from the definition; target, draft float64 arrays."""
    one = 1 << 36

    def whole(p):
        p = 0.0 if math.isnan(p) else min(max(p, 0.0), 1.0)
        return int(p * one)                       # exact: a power of two

    V = target.shape[1]
    accepted, nxt = [], []
    for r in range(len(off) - 1):
        s, n = int(off[r + 1] - off[r]), 0
        while n < s:
            d = int(off[r]) + n
            x = int(ids[d])
            if not 0 <= x < V:
                break
            q = one if draft is None else whole(draft[d, x])
            if not int(u[d] * 2 ** 24) * q < whole(target[d + r, x]) << 24:
                break
            n += 1
        p = [whole(float(v)) for v in target[int(off[r]) + r + n]]
        w = p
        if n < s:
            d = int(off[r]) + n
            q = [whole(float(v)) for v in draft[d]] if draft is not None else [one if v == ids[d] else 0 for v in range(V)]
            w = [max(a - b, 0) for a, b in zip(p, q)]
            if sum(w) == 0:
                w = p
        S = sum(w)
        t = int(u_next[r] * 2 ** 24) * S >> 24
        token, run = -1, 0
        if S:
            for v, x in enumerate(w):
                run += x
                if run > t:
                    token = v
                    break
        accepted.append(n)
        nxt.append(token)
    return np.array(accepted, np.int32), np.array(nxt, np.int32)
