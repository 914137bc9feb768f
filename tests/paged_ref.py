"""Plain references, in 64 bits, of the paged-cache and sampling operators
(test infrastructure)."""
import math

import numpy as np

PAGE = 64


def e4m3_table():
    """The value of each of the 256 e4m3 codes (OCP FP8 E4M3, bias 7)."""
    v = np.empty(256)
    for c in range(256):
        s, e, m = -1.0 if c & 128 else 1.0, (c >> 3) & 15, c & 7
        v[c] = s * (m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
        if c & 127 == 127:
            v[c] = np.nan
    return v


TABLE = e4m3_table()


def to_e4m3(x):
    """float64 -> e4m3 codes: nearest, halves to the even code, at most 448 in size, NaN kept."""
    x = np.asarray(x, dtype=np.float64)
    a = np.minimum(np.abs(x), 448.0)
    pos = TABLE[:127]                                   # 0 .. 448, increasing with the code
    hi = np.clip(np.searchsorted(pos, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    down, up = a - pos[lo], pos[hi] - a
    code = np.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
    code = np.where(np.isnan(x), 127, code).astype(np.uint8)
    return np.where(np.signbit(x), code | 128, code).astype(np.uint8)


def scale_of(amax):
    """2^e, least e in [-40, 120] with amax <= 448 2^e."""
    e = -40
    while e < 120 and amax > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def page_assign(seq_len, grow, table, free, count, max_slots):
    """One request after the other; returns (new_len, table, free stack, count, slots, start, flag)."""
    table, free = table.copy(), list(free[:count])
    pages = lambda n: -(-n // PAGE)
    row = table.shape[1] * PAGE
    flag, new_len, slots, start = 0, [], [], [0]
    B = len(seq_len)
    for b in range(B):
        if grow[b] <= 0:
            new = max(0, seq_len[b] + grow[b])
            free += list(table[b, pages(new):pages(seq_len[b])])
    need_pages = need_slots = 0
    at_start = len(free)
    for b in range(B):
        old = int(seq_len[b])
        if grow[b] <= 0:
            new_len.append(max(0, old + int(grow[b])))
        elif old + grow[b] > row:
            flag |= 1
            new_len.append(old)
        else:
            need = pages(old + grow[b]) - pages(old)
            need_pages += need
            need_slots += grow[b]
            if (need and need_pages > at_start) or need_slots > max_slots:
                flag |= 1
                new_len.append(old)
            else:
                for j in range(need):
                    table[b, pages(old) + j] = free.pop()
                slots += [table[b, t // PAGE] * PAGE + t % PAGE for t in range(old, old + int(grow[b]))]
                new_len.append(old + int(grow[b]))
        start.append(len(slots))
    return new_len, table, free, len(free), slots, start, flag


def append(codes, scales, new, slots, start):
    """codes [R][L][N][H][64][D] uint8, scales [R][L][N][H], new float64 [R][L][B][W][H][D]:
    copies with the first start[b+1] - start[b] tokens of each sequence stored."""
    codes, scales = codes.copy(), scales.copy()
    R, L, _, H = scales.shape
    for b in range(len(start) - 1):
        t = start[b]
        while t < start[b + 1]:
            page, at = divmod(int(slots[t]), PAGE)
            n = min(PAGE - at, start[b + 1] - t)
            for r in range(R):
                for l in range(L):
                    for h in range(H):
                        x = new[r, l, b, t - start[b]:t - start[b] + n, h]
                        fin = np.abs(x[np.isfinite(x)])
                        s = scale_of(fin.max(initial=0.0))
                        if at:
                            held = float(scales[r, l, page, h])
                            s = max(s, held)
                            if s != held:
                                codes[r, l, page, h, :at] = to_e4m3(TABLE[codes[r, l, page, h, :at]] * (held / s))
                        codes[r, l, page, h, at:at + n] = to_e4m3(x / s)
                        scales[r, l, page, h] = s
            t += n
    return codes, scales


def attention(k, ks, v, vs, table, P, T, q, kb, vb, scale=None, masked=()):
    """k, v codes [N][H][64][D] of the slabs read, ks, vs [N][H]; q [B][T][Hq][D], kb, vb
    [B][T][H][D] float64.  masked: (b, tile) pairs whose keys are hidden.  (out, lse)."""
    B, Tm, Hq, D = q.shape
    H = kb.shape[2]
    G = Hq // H
    scale = 1 / math.sqrt(D) if scale is None else scale
    out, lse = np.zeros((B, Tm, Hq, D)), np.full((B, Hq, Tm), -np.inf)
    for b in range(B):
        tiles = [t for t in range(-(-int(P[b]) // PAGE)) if (b, t) not in masked]
        for h in range(H):
            K, V = [], []
            for t in tiles:
                n = min(PAGE, int(P[b]) - t * PAGE)
                pg = table[b, t]
                K.append(TABLE[k[pg, h, :n]] * float(ks[pg, h]))
                V.append(TABLE[v[pg, h, :n]] * float(vs[pg, h]))
            for i in range(int(T[b])):
                keys = np.concatenate(K + [kb[b, :i + 1, h]])
                vals = np.concatenate(V + [vb[b, :i + 1, h]])
                s = q[b, i, h * G:(h + 1) * G] @ keys.T * scale
                m = s.max(1, keepdims=True)
                w = np.exp(s - m)
                l = w.sum(1, keepdims=True)
                out[b, i, h * G:(h + 1) * G] = w @ vals / l
                lse[b, h * G:(h + 1) * G, i] = (m + np.log(l))[:, 0]
    return out, lse


def sample_row(logits, e, T, k, p, min_p, u):
    """One draw in whole numbers.  logits: the row as float64 (NaN allowed); e: the binary32 e_v of
    the row at this temperature (float64 array); returns (token, R, kept)."""
    x = np.where(np.isnan(logits), -np.inf, logits)
    m = x.max()
    if m == -np.inf:
        return -1, 0, np.zeros(len(x), bool)
    greedy = not T > 0
    w = [int(round(float(t) * 2.0 ** 32)) for t in (np.where(x == m, 1.0, 0.0) if greedy else e)]
    order = np.argsort(-x, kind="stable")
    if greedy:
        order = order[:1]
    elif 0 < k < len(x):
        order = order[:k]
    if p < 1:
        S = sum(w[i] for i in order)
        target = min(max(1, int(math.ceil(float(p) * float(S)))), S)
        run, n = 0, 0
        while run < target:
            run += w[order[n]]
            n += 1
        order = order[:n]
    if min_p > 0:
        order = [i for i in order if x[i] == m or e[i] >= min(min_p, 1.0)]
    kept = np.zeros(len(x), bool)
    kept[list(order)] = True
    R = sum(w[i] for i in order)
    r = min(int(math.floor(float(u) * float(R))), R - 1)
    run = 0
    for i in np.flatnonzero(kept):
        run += w[i]
        if run > r:
            return int(i), R, kept
