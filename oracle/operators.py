"""Oracle of the operators on a paged layer: numpy, from the definitions, element by element of a pool's
logical form [block][slot][head][dim].  Shares no code with the library.

append_rows follows the definition in the arithmetic it states (fp32, each product, sum and quotient rounded
once), so codes can be compared for equality; attend and rotate64 are in 64 bits."""
import numpy as np

TOP = {"e4m3": np.float32(448), "int8": np.float32(127)}


def e4m3_values():
    """The 256 codes' values: sign, 4 exponent bits (bias 7), 3 fraction bits; 0x7f and 0xff are NaN."""
    c = np.arange(256)
    e, f = (c >> 3) & 15, c & 7
    v = np.where(e == 0, f / 8.0 * 2.0 ** -6, (1 + f / 8.0) * 2.0 ** (e - 7.0))
    v[(c & 0x7f) == 0x7f] = np.nan
    return np.where(c & 0x80, -v, v)


_POS = e4m3_values()[:0x7f]  # ascending magnitudes of the codes 0 .. 0x7e


def e4m3_round(x):
    """Codes of x (any float array), to nearest even, magnitudes above 448 to 448."""
    x = np.asarray(x, dtype=np.float64)
    a = np.minimum(np.abs(x), 448.0)
    hi = np.clip(np.searchsorted(_POS, a), 1, 0x7e)
    lo = hi - 1
    mid = (_POS[lo] + _POS[hi]) / 2
    up = (a > mid) | ((a == mid) & (hi % 2 == 0))
    return (np.where(up, hi, lo) | np.where(np.signbit(x), 0x80, 0)).astype(np.uint8)


def partners(rot, interleaved):
    """Index of the first and second element of every rotated pair."""
    j = np.arange(rot // 2)
    return (2 * j, 2 * j + 1) if interleaved else (j, j + rot // 2)


def rotate(x, cos, sin, interleaved):
    """x [n, heads, D] and tables [n, rot/2], all of one float type, in that type's arithmetic."""
    y = x.copy()
    i, k = partners(2 * cos.shape[1], interleaved)
    c, s = cos[:, None, :], sin[:, None, :]
    y[..., i] = x[..., i] * c - x[..., k] * s
    y[..., k] = x[..., k] * c + x[..., i] * s
    return y


def quantise(y, kind):
    """(codes uint8 / int8, scales fp32) of fp32 rows."""
    assert y.dtype == np.float32
    with np.errstate(all="ignore"):
        most = np.abs(y).max(-1)
        finite = np.isfinite(y).all(-1)
        scale = (most / TOP[kind]).astype(np.float32)
        scale = np.where(scale < np.float32(2.0 ** -126), np.float32(0), scale)
        scale = np.where(finite, scale, np.float32(np.nan))
        some = (scale > 0)[..., None]
        z = np.where(some, y / np.where(some, scale[..., None], 1).astype(np.float32), np.float32(0)).astype(np.float32)
        codes = e4m3_round(z) if kind == "e4m3" else np.rint(z).astype(np.int8)
    return codes, scale


def values(codes, scales, kind):
    """What a quantised row stands for, in 64 bits."""
    v = e4m3_values()[codes.view(np.uint8)] if kind == "e4m3" else codes.astype(np.float64)
    return v * scales[..., None].astype(np.float64)


def attend(q, keys, vals, scale):
    """One request: q [Hq, D], keys and vals [n, H, D], all 64 bits -> (out [Hq, D], lse [Hq], sum of weights * |v|)."""
    Hq, D = q.shape
    n, H, _ = keys.shape
    out, lse, mass = np.zeros((Hq, D)), np.full(Hq, -np.inf), np.zeros((Hq, D))
    for h in range(Hq):
        if n == 0:
            continue
        k, v = keys[:, h // (Hq // H)], vals[:, h // (Hq // H)]
        s = k @ q[h] * scale
        m = s.max()
        if m == -np.inf:
            continue
        e = np.exp(s - m)
        out[h], mass[h] = e @ v / e.sum(), e @ np.abs(v) / e.sum()
        lse[h] = m + np.log(e.sum())
    return out, lse, mass


def attend_chunk(q, keys, vals, scale, window=0, sinks=0, there=None):
    """One request's new tokens, the last len(q) of its len(keys): q [n, Hq, D], keys and vals [len, H, D], all 64 bits; row i sees
    keys j <= p = len - n + i, with a window j > p - window or j < sinks; there [len]: keys that can be seen at all.
    -> (out [n, Hq, D], lse [n, Hq], weights [n, Hq, len])."""
    n, Hq, D = q.shape
    total, H, _ = keys.shape
    j, p = np.arange(total), np.arange(total - n, total)[:, None]
    seen = (j <= p) & ((window == 0) | (j > p - window) | (j < sinks))
    if there is not None:
        seen &= there
    out, lse, weights = np.zeros((n, Hq, D)), np.full((n, Hq), -np.inf), np.zeros((n, Hq, total))
    for h in range(Hq):
        k, v = keys[:, h // (Hq // H)], vals[:, h // (Hq // H)]
        with np.errstate(invalid="ignore"):
            s = np.where(seen, q[:, h] @ k.T * scale, -np.inf)
            m = s.max(1)
            e = np.exp(s - np.where(m == -np.inf, 0, m)[:, None])  # NaN in rows with a score that is NaN or infinite
            total_e = e.sum(1)
            w = e / np.where(total_e == 0, 1, total_e)[:, None]
            some = total_e != 0
            # a key that is not seen has no part, whatever its value is, and no key has where none has any weight
            bad = ~np.isfinite(v).all(1)
            out[:, h] = w @ np.where(bad[:, None], 0, v)
            for x in np.flatnonzero(bad):
                out[seen[:, x] & some, h] += w[seen[:, x] & some, x][:, None] * v[x]
            lse[some, h] = m[some] + np.log(total_e[some])
        weights[:, h] = w
    return out, lse, weights
