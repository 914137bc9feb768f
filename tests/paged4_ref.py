"""Plain references, in 64 bits, of the 4-bit cache's operators, of norm and rotation, and of
speculative acceptance (test infrastructure)."""
import math
from fractions import Fraction

import numpy as np

from tests import paged_ref

PAGE, GROUP = 64, 32


def scale_table():
    """What each of the 256 scale bytes stands for: the binary16 number of the bits byte << 7."""
    v = np.empty(256)
    for b in range(256):
        e, m = b >> 3, b & 7
        v[b] = m * 2.0 ** -17 if e == 0 else (8 + m) * 2.0 ** (e - 18)
        if e == 31:
            v[b] = np.inf if m == 0 else np.nan
    return v


SCALES = scale_table()


def quantise(x, unit):
    """Codes (1 to 15) and scale bytes of float64 values [..., D]."""
    g = x.reshape(x.shape[:-1] + (-1, GROUP))
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        m = np.where(np.isfinite(g), np.abs(g), 0.0).max(-1) / unit
        t = (m.astype(np.float32) * np.float32(1 / 7)).astype(np.float64)   # as defined: in binary32
        e = np.floor(np.log2(np.where((t > 0) & np.isfinite(t), t, 1.0)))
        e = np.where(2.0 ** e > t, e - 1, np.where(2.0 ** (e + 1) <= t, e + 1, e))   # 2^e <= t < 2^(e + 1)
        step = 2.0 ** np.maximum(e - 3, -17)
        s = np.minimum(np.where(np.isfinite(t), np.rint(t / step) * step, 60.0), 60.0)
        byte = np.searchsorted(SCALES[:168], s)
        assert np.array_equal(SCALES[byte], s)
        code = np.rint(g / np.where(s > 0, s * unit, 1.0)[..., None])
        code = np.where((s > 0)[..., None], np.clip(np.nan_to_num(code, posinf=7, neginf=-7), -7, 7), 0)
    byte = np.where(np.isnan(g).any(-1), 255, byte)
    return (code + 8).astype(np.uint8).reshape(x.shape), byte.astype(np.uint8)


def append(k, ks, v, vs, ku, vu, kn, vn, slots, start):
    """Copies of a cache's codes and scales ([R][L][N][H]...) with the tokens stored; ku, vu [R][L][H]."""
    k, ks, v, vs = (a.copy() for a in (k, ks, v, vs))
    for b in range(len(start) - 1):
        for j in range(start[b], start[b + 1]):
            page, t = divmod(int(slots[j]), PAGE)
            c, s = quantise(kn[:, :, b, j - start[b]], ku[..., None])                  # [R][L][H][D], [R][L][H][D / 32]
            k[:, :, page, :, t], ks[:, :, page, :, t] = c[..., 0::2] | c[..., 1::2] << 4, s
            c, s = quantise(vn[:, :, b, j - start[b]], vu[..., None])
            word = v[:, :, page, :, t // 8, :, t % 8 // 2]
            v[:, :, page, :, t // 8, :, t % 8 // 2] = word & (0xf0 if t % 2 == 0 else 0x0f) | c << 4 * (t % 2)
            vs[:, :, page, :, :, t] = s
    return k, ks, v, vs


def keys(k, ks, unit):
    """float64 [..., H, 64, D] of codes [..., H, 64, D / 2]; unit [H]."""
    c = np.stack([k & 15, k >> 4], -1).reshape(k.shape[:-1] + (-1,)).astype(np.float64) - 8
    return c * np.repeat(SCALES[ks], GROUP, -1) * unit[:, None, None]


def values(v, vs, unit):
    """float64 [..., H, 64, D] of codes [..., H, 8, D, 4]."""
    c = np.stack([v & 15, v >> 4], -1).reshape(v.shape[:-1] + (8,)).astype(np.float64) - 8   # [..., 8, D, 8]
    c = np.swapaxes(c, -1, -2)
    c = c.reshape(c.shape[:-3] + (PAGE, c.shape[-1]))
    return c * np.repeat(np.swapaxes(SCALES[vs], -1, -2), GROUP, -1) * unit[:, None, None]


def attention(K, V, table, P, T, q, kb, vb, scale=None, masked=()):
    """K, V float64 [N][H][64][D]; the rest as paged_ref.attention.  (out, lse, and the weighted mean distance of
    the values from the output, by which an error of the weights moves it)."""
    B, Tm, Hq, D = q.shape
    H = kb.shape[2]
    G = Hq // H
    scale = 1 / math.sqrt(D) if scale is None else scale
    out, lse, dev = np.zeros((B, Tm, Hq, D)), np.full((B, Hq, Tm), -np.inf), np.zeros((B, Tm, Hq, D))
    for b in range(B):
        tiles = [(table[b, t], min(PAGE, int(P[b]) - t * PAGE)) for t in range(-(-int(P[b]) // PAGE))
                 if (b, t) not in masked]
        for h in range(H):
            pk = np.concatenate([K[pg, h, :n] for pg, n in tiles] + [kb[b, :0, h]])
            pv = np.concatenate([V[pg, h, :n] for pg, n in tiles] + [vb[b, :0, h]])
            for i in range(int(T[b])):
                k, v = np.concatenate([pk, kb[b, :i + 1, h]]), np.concatenate([pv, vb[b, :i + 1, h]])
                s = q[b, i, h * G:(h + 1) * G] @ k.T * scale
                m = s.max(1, keepdims=True)
                w = np.exp(s - m)
                l = w.sum(1, keepdims=True)
                o = w @ v / l
                out[b, i, h * G:(h + 1) * G] = o
                lse[b, h * G:(h + 1) * G, i] = (m + np.log(l))[:, 0]
                for g in range(G):
                    dev[b, i, h * G + g] = w[g] @ np.abs(v - o[g]) / l[g]
    return out, lse, dev


TWO_PI = 2 * Fraction(314159265358979323846264338327950288419716939937510, 10 ** 50)


def angles(place, freq):
    """float64 angles place * freq modulo 2 pi: [...] x [n], exact to 2^-52."""
    out = np.empty(np.shape(place) + (len(freq),))
    for at in np.ndindex(np.shape(place)):
        for j, f in enumerate(freq):
            t = int(place[at]) * Fraction(float(f)) / TWO_PI
            out[at + (j,)] = float((t - round(t)) * TWO_PI)
    return out


def norm_rope(x, weight, eps, angle, interleaved):
    """x float64 [B][T][H][D], angle [B][T][rd / 2]; also the size that errors go by."""
    if eps is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * (1.0 if weight is None else weight)
    n = angle.shape[-1]
    y, size = x.copy(), np.abs(x)
    a, c = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    cos, sin = np.cos(angle)[:, :, None], np.sin(angle)[:, :, None]
    y[..., a] = x[..., a] * cos - x[..., c] * sin
    y[..., c] = x[..., c] * cos + x[..., a] * sin
    size[..., a] = size[..., c] = np.abs(x[..., a]) + np.abs(x[..., c])
    return y, size


def probabilities(logits, e, T, k, p, min_p):
    """Binary32 probabilities of a row, its whole-number weights and their sum."""
    x = np.where(np.isnan(logits), -np.inf, logits)
    _, R, kept = paged_ref.sample_row(logits, e, T, k, p, min_p, 0.0)
    if not T > 0:
        e = np.where(x == x.max(), 1.0, 0.0)
    e = np.where(kept, e, 0.0).astype(np.float32)
    inv = np.float32(1.0) / np.float32(R / 2.0 ** 32) if R else np.float32(0)
    return e * inv, [int(round(float(t) * 2.0 ** 32)) for t in e], R


def draw(weights, u):
    S = sum(weights)
    u = float(u) if u >= 0 else 0.0
    r = min(int(math.floor(u * float(S))), S - 1)
    run = 0
    for v, w in enumerate(weights):
        run += w
        if run > r:
            return v
    return -1


def speculative(target, drafter, ids, u, again):
    """One sequence: target and drafter are lists of (p, weights, R) for its places.  (accepted, next)."""
    W = len(target)
    for i in range(W):
        p, w, _ = target[i]
        q = drafter[i][0]
        y = int(ids[i])
        if 0 <= y < len(p) and float(u[i]) * float(q[y]) < float(p[y]):
            continue
        with np.errstate(over="ignore"):
            rest = [int(round(float(x) * 2.0 ** 40)) for x in np.maximum(p - q, np.float32(0))]
        return i, draw(rest if sum(rest) else w, again)
    return W, int(ids[W - 1])
