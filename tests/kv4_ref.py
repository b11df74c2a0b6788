"""Definition of the 4-bit KV cache in 64 bits (numpy), for its tests: the
microscaled form, the byte order of a record and attention over its values."""
import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def bf16(x):
    """float64 values of x rounded to bf16, half to even."""
    b = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32)
    r = ((b + 0x7FFF + ((b >> 16) & 1)) >> 16 << 16).astype(np.uint32)
    return np.where(np.isfinite(x), r.view(np.float32), np.float32(x)).astype(np.float64)


def quantise(x):
    """Codes [..., hd] and scale bytes [..., hd/32] of rows x (float64)."""
    b = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    bad = ~np.isfinite(b).all(-1)
    amax = np.abs(np.where(bad[..., None], 0.0, b)).max(-1)
    e = np.maximum(np.frexp(amax)[1] - 1 - 2, -125)
    e = np.where(amax == 0, -125, e)
    y = np.abs(np.where(bad[..., None], 0.0, b)) / np.exp2(e.astype(np.float64))[..., None]
    gap = np.abs(y[..., None] - E2M1)  # exact: y and the grid have few bits
    near = gap == gap.min(-1, keepdims=True)
    code = np.where(near.sum(-1) == 1, near.argmax(-1),
                    np.where(near.argmax(-1) % 2 == 0, near.argmax(-1), near.argmax(-1) + 1))  # ties: the even code
    code = np.where(bad[..., None], 0, code + 8 * np.signbit(b))
    return code.astype(np.uint8).reshape(x.shape), np.where(bad, 255, e + 127).astype(np.uint8)


def values(code, scale):
    x = np.where(code < 8, 1.0, -1.0) * E2M1[code & 7]
    s = np.exp2(scale.astype(np.float64) - 127)
    s = np.where(scale == 255, np.nan, s)
    return (x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32) * s[..., None]).reshape(x.shape)


def rotate(k, cos, sin, pos):
    """k [T][Hkv][hd] (float64), rotated and rounded to fp32 once."""
    h = k.shape[-1] // 2
    c, s = (t.astype(np.float64)[np.clip(pos, 0, len(cos) - 1)][:, None] for t in (cos, sin))
    out = np.concatenate([k[..., :h] * c - k[..., h:] * s, k[..., h:] * c + k[..., :h] * s], -1)
    out = out.astype(np.float32).astype(np.float64)
    out[(pos < 0) | (pos >= len(cos))] = np.nan
    return out


def _places(hd):
    """Byte offsets in a record for (slot, d): key code, value code (+ their
    high-nibble flags), and for (slot, block): key scale, value scale."""
    s, d, b = np.arange(32)[:, None], np.arange(hd)[None, :], np.arange(hd // 32)[None, :]
    i, half, j = s // 8, s // 4 % 2, s % 4
    g, rest, u = d // (hd // 4), d % (hd // 4), hd // 32
    kc = ((((half * 4 + g) * 4 + i) * 4 + j) * u + rest // 8) * 4 + rest % 8 // 2
    w = 512 // hd
    t, r = d % 32 // w, d % w
    vc = 16 * hd + ((((t // 4) * 4 + s // 8) * u + d // 32) * w + r) * 16 + (t // 2 % 2) * 8 + s % 8
    ks = 32 * hd + ((b * 4 + i) * 4 + j) * 2 + half
    vs = 33 * hd + b * 32 + s
    return kc, np.broadcast_to(d % 2, kc.shape), vc, np.broadcast_to(t % 2, vc.shape), ks, vs


def pack(k4, v4, cap, fill=None):
    """Records [Hkv][cap/32][34 hd] of quantised rows ([Hkv][n][..] codes and
    scale bytes, slots 0 .. n - 1); fill: the bytes before them."""
    (kc, ks), (vc, vs) = k4, v4
    H, n, hd = kc.shape
    rec = np.zeros((H, cap // 32, 34 * hd), np.uint8) if fill is None else fill.copy()
    pk, hk, pv, hv, pks, pvs = _places(hd)
    for t in range((n + 31) // 32):
        m = min(32, n - 32 * t)
        at = slice(32 * t, 32 * t + m)
        out = rec[:, t]
        for c, p, hi in ((kc, pk, hk), (vc, pv, hv)):
            for nib in (0, 1):
                sel = hi[:m] == nib
                cur = out[:, p[:m][sel]]
                new = c[:, at][:, sel]
                out[:, p[:m][sel]] = (cur & 0x0F) | (new << 4) if nib else (cur & 0xF0) | new
        out[:, pks[:m]] = ks[:, at]
        out[:, pvs[:m]] = vs[:, at]
    return rec


def visible(T, n_tree, Lc, masks, sink, window):
    """[T][Lc + n_tree] booleans; masks: [T] python integers."""
    see = np.zeros((T, Lc + n_tree), bool)
    see[:, max(0, Lc - window) if window else 0 : Lc] = True
    if window:
        see[:, : min(sink, Lc)] = True
    for t in range(T):
        for j in range(n_tree):
            see[t, Lc + j] = masks[t] >> j & 1
    return see


def attention(q, k, v, see):
    """q [T][H][hd], k, v [Hkv][n][hd]: (output [T][H hd], its bound's scales:
    sum of p |v| per element and the largest sum of |q k| per row)."""
    T, H, hd = q.shape
    G = H // k.shape[0]
    out, size = np.zeros((T, H, hd)), np.zeros((T, H, hd))
    mass = np.zeros((T, H))
    for h in range(H):
        for t in range(T):
            on = see[t]
            if not on.any():
                continue
            kk, vv = k[h // G][on], v[h // G][on]
            x = kk @ q[t, h] / np.sqrt(hd)
            p = np.exp(x - x.max())
            p /= p.sum()
            out[t, h], size[t, h] = p @ vv, p @ np.abs(vv)
            mass[t, h] = (np.abs(kk) @ np.abs(q[t, h])).max() / np.sqrt(hd)
    return out.reshape(T, -1), size.reshape(T, -1), mass


def bound(ref, size, mass, hd, n):
    """Largest error of a bf16 output with bf16 probabilities (each rounding at
    most 2^-8 of its value) and fp32 scores and sums: a score of hd terms is off
    by at most (hd + 4) 2^-24 of its terms' sum, which moves every probability
    and the sum they are divided by by as much; a sum of n terms in runs of 32
    by (n / 32 + 64) 2^-24 of theirs; the exponent's own steps by 2^-18."""
    per = np.repeat(2 * (hd + 4) * 2.0**-24 * mass, hd, axis=1) + (n / 32 + 64) * 2.0**-23 + 2.0**-18
    return 2.0**-8 * np.abs(ref) * (1 + 2.0**-7) + size * (2.0**-8 + per) * (1 + 2.0**-7) + 1e-37
