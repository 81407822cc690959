"""The 8-bit cache and attention over it from their definitions, in 64 bits (numpy)."""
import numpy as np


def values(x):
    """What the cache holds in the place of vectors x [..., head_dim] (float32): e4m3 codes of x / 2^e times 2^e, e the smallest exponent, not below
    -126, with max |x| <= 448 * 2^e; entries that are not finite have no part in e and become no numbers."""
    x = np.asarray(x, dtype=np.float32).astype(np.float64)
    fine = np.isfinite(x)
    e = exponents(x)
    y = np.where(fine, x, 0.0) / np.exp2(e)[..., None]
    assert np.all(np.abs(y) <= 448.0)
    lead = np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -6)))     # of the leading bit, that of the smallest normal code at least
    step = np.exp2(lead - 3)
    return np.where(fine, np.rint(y / step) * step * np.exp2(e)[..., None], np.nan)


def exponents(x):
    x = np.asarray(x, dtype=np.float32).astype(np.float64)
    top = np.where(np.isfinite(x), np.abs(x), 0.0).max(axis=-1)
    mant, ex = np.frexp(top)                                         # top = mant * 2^ex, mant in [1/2, 1)
    e = np.where(top > 0, ex - 9 + (mant > 0.875), -126)             # 448 = 0.875 * 2^9
    return np.maximum(e, -126).astype(np.float64)


def attend(q, k, v, pos):
    """(out [m, Hq * dh], bound) of float arrays q [m, Hq, dh], k, v [n, Hkv, dh].

    The bound per row: queries are held to 2^-22 of themselves, products of codes are exact and their sums over head_dim, like the three
    multiplications by scales, are off by 2^-24 per operation at most; an error d of the scores changes the weights by a factor within exp(+-2d), and sums of
    weights and of weighted values over n positions (chains of at most 16 + n / 256 / 16 + 512 additions, and the two parts of a probability, 2^-22) add 2^-22 * 40 or less
    for the lengths used here."""
    m, Hq, dh = q.shape
    G = Hq // k.shape[1]
    q, k, v = (np.asarray(a, dtype=np.float64) for a in (q, k, v))
    out, bound = np.zeros((m, Hq, dh)), np.zeros((m, Hq, dh))
    for r in range(m):
        kr, vr = k[: pos[r] + 1], v[: pos[r] + 1]
        for h in range(Hq):
            kk, vv = kr[:, h // G], vr[:, h // G]
            s = kk @ q[r, h] / np.sqrt(dh)
            size = np.max(np.abs(kk) @ np.abs(q[r, h])) / np.sqrt(dh)
            d = size * (2.0 ** -22 + (dh + 4) * 2.0 ** -24) + np.max(np.abs(s)) * 2.0 ** -22
            p = np.exp(s - s.max())
            p /= p.sum()
            out[r, h] = p @ vv
            bound[r, h] = (p @ np.abs(vv)) * (np.expm1(2 * d) + 2.0 ** -22 * 40) + 1e-38
    return out.reshape(m, Hq * dh), bound.reshape(m, Hq * dh)
