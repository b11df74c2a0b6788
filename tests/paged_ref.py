"""Definition of the paged KV cache in 64 bits (numpy), for its tests: the order
of a tile, where slots lie, and attention over them with its error bound."""
import numpy as np


def key_places(hd):
    """[32][hd]: places of a tile's keys, [2 h][hd/32 u][4 g][4 i][4 j][8 e] with
    slot 8i + 4h + j and element g hd/4 + 8u + e."""
    sl, d = np.arange(32)[:, None], np.arange(hd)[None]
    i, h, j = sl // 8, sl // 4 % 2, sl % 4
    g, u, e = d // (hd // 4), d % (hd // 4) // 8, d % 8
    return ((((h * (hd // 32) + u) * 4 + g) * 4 + i) * 4 + j) * 8 + e


def value_places(hd):
    """[32][hd]: places of a tile's values, [hd/16 m][4 g][16 r][8 e] with slot
    8g + e and element 16m + r."""
    sl, d = np.arange(32)[:, None], np.arange(hd)[None]
    return ((d // 16 * 4 + sl // 8) * 16 + d % 16) * 8 + sl % 8


def put(pages, hd, page, table, slot, k, v):
    """Keys and values k, v [Hkv][hd] into a slot of pages [n][2][Hkv][page * hd]."""
    p, t = table[slot // page], slot % page // 32 * 32 * hd
    pages[p, 0][:, t + key_places(hd)[slot % 32]] = k
    pages[p, 1][:, t + value_places(hd)[slot % 32]] = v


def rotate(x, cos, sin, pos):
    """x [T][H][hd] (float64) rotated by its positions, not rounded."""
    h = x.shape[-1] // 2
    c, s = (t.astype(np.float64)[np.clip(pos, 0, len(cos) - 1)][:, None] for t in (cos, sin))
    out = np.concatenate([x[..., :h] * c - x[..., h:] * s, x[..., h:] * c + x[..., :h] * s], -1)
    out[(pos < 0) | (pos >= len(cos))] = np.nan
    return out


def rotate_bound(x, ref):
    """Largest error of the bf16 rotation of bf16 values by fp32 angles: two
    fp32 steps (a product, the fused sum) of terms of at most |x0| + |x1|, then
    half a step of bf16."""
    h = x.shape[-1] // 2
    terms = np.abs(x[..., :h]) + np.abs(x[..., h:])
    return np.concatenate([terms, terms], -1) * 2.0**-23 * (1 + 2.0**-7) + np.abs(ref) * 2.0**-8 + 1e-40


def visible(T, Lc, nodes, masks, sink, window):
    """[T][Lc + nodes + T] booleans; masks: None (causal) or [T] python integers."""
    n = Lc + nodes + T
    see = np.zeros((T, n), bool)
    for t in range(T):
        end = Lc if masks else Lc + nodes + t  # the slots that the window counts
        see[t, (max(0, end - window) if window else 0) : end] = True
        if window:
            see[t, : min(sink, end)] = True
        if masks:
            for j in range(n - Lc):
                see[t, Lc + j] = masks[t] >> j & 1
        else:
            see[t, end] = True
    return see


def attention(q, k, v, see):
    """q [T][H][hd], k, v [Hkv][n][hd]: the output [T][H][hd] and the largest
    error of one in bf16.  With weights p (their sum 1): a probability is
    rounded to bf16 (2^-8 of itself) and so is the sum they are divided by, and
    a score of hd terms is off by at most (hd + 4) 2^-24 of its terms' sum, the
    exponential by 2^-18: each weight moves by d, |d| <= 2^-8 + 2 (hd + 4) 2^-24
    mass + 2^-18, and the output by sum p d (v - o) <= max d (sum p |v| + |o|).
    Sums of n terms in runs of 32 and their joins: (n / 32 + 64) 2^-23 of their
    terms.  The output's own rounding: 2^-8."""
    T, H, hd = q.shape
    G, n = H // k.shape[0], see.shape[1]
    out, err = np.zeros((T, H, hd)), np.zeros((T, H, hd))
    for h in range(H):
        kk, vv = k[h // G], v[h // G]
        x = np.where(see, q[:, h] @ kk.T / np.sqrt(hd), -np.inf)
        top = x.max(1, keepdims=True)
        p = np.exp(x - np.where(np.isfinite(top), top, 0))
        p /= np.maximum(p.sum(1, keepdims=True), 1e-300)
        o, size = p @ vv, p @ np.abs(vv)
        mass = np.where(see, np.abs(q[:, h]) @ np.abs(kk).T, 0).max(1, keepdims=True) / np.sqrt(hd)
        d = 2.0**-8 + 2 * (hd + 4) * 2.0**-24 * mass + 2.0**-18
        out[:, h] = o
        err[:, h] = (d * (size + np.abs(o)) + (n / 32 + 64) * 2.0**-23 * size + 2.0**-8 * np.abs(o)) * (1 + 2.0**-6) + 1e-37
    return out, err
