"""Paged-cache operators in float64: head norms with rotary positions, the 8-bit rows, page choice and attention of new
rows over the pages.  Written from the formulas, one sequence and head at a time."""

import numpy as np


def qk_norm_rope_ref(x, w, eps, pos, base):
    """x [T, H, d], w [d] or None, pos [T]; rotate-half pairs (i, i + d/2), frequencies base^(-2i/d); base 0: none."""
    x = np.asarray(x, np.float64)
    d = x.shape[-1]
    if w is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(w, np.float64)
    if base:
        h = d // 2
        a = np.asarray(pos, np.float64)[:, None] * base ** (-2.0 * np.arange(h) / d)
        c, s = np.cos(a)[:, None], np.sin(a)[:, None]
        lo, hi = x[..., :h], x[..., h:]
        x = np.concatenate([lo * c - hi * s, hi * c + lo * s], -1)
    return x


# The values of an E4M3 byte: sign, 4 exponent bits (bias 7), 3 mantissa bits; 0x7F is NaN.
def _e4m3_values():
    out = np.empty(256)
    for i in range(256):
        e, m = (i >> 3) & 15, i & 7
        v = (m / 8) * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        if e == 15 and m == 7:
            v = np.nan
        out[i] = -v if i & 128 else v
    return out


E4M3 = _e4m3_values()


def e4m3_round(x):
    """x (|x| <= 448 or NaN) to the nearest E4M3 value, ties to the even mantissa."""
    x = np.asarray(x, np.float64)
    pos = E4M3[:127]
    a = np.abs(x)
    hi = np.clip(np.searchsorted(pos, np.nan_to_num(a)), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - pos[lo], pos[hi] - a
    take_hi = (dh < dl) | ((dh == dl) & (hi % 2 == 0))
    v = np.where(take_hi, pos[hi], pos[lo])
    return np.where(np.isnan(x), np.nan, np.where(np.signbit(x), -v, v))


def quantise_ref(x):
    """Rows [..., d] to (E4M3 values, exponents): e least with max|x| <= 448 * 2^e over the finite elements."""
    x = np.asarray(x, np.float64)
    a = np.where(np.isfinite(x), np.abs(x), 0).max(-1)
    e = np.full(a.shape, -100)
    while np.any(short := (e < 120) & (a > 448.0 * 2.0 ** e.astype(np.float64))):
        e[short] += 1
    y = np.where(np.isfinite(x), x, np.nan) * 2.0 ** -e[..., None].astype(np.float64)
    return e4m3_round(y), e


# The values of the codes 0..7 of E2M1; 8..15 are their negatives.
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def e2m1_codes(x):
    """x (|x| <= 6) to the code of the nearest E2M1 value, ties to the even code."""
    x = np.asarray(x, np.float64)
    a = np.abs(x)[..., None]
    off = np.abs(a - E2M1)
    code = np.argmin(off + 1e-9 * (np.arange(8) % 2), -1)     # neighbours are equally far at a border, and one is even
    return code + 8 * np.signbit(x)


def quantise4_ref(x):
    """Rows [..., d] to (codes [..., d], exponents [..., d / 32]): e least with max|x| <= 6 * 2^e over 32 channels; a group
    with an element that is not finite has exponent 128 (its byte is 255)."""
    x = np.asarray(x, np.float64)
    x = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    bad = ~np.isfinite(x).all(-1)
    x = np.where(np.isfinite(x), x, 0)
    a = np.abs(x).max(-1)
    e = np.full(a.shape, -100)
    while np.any(short := (e < 126) & (a > 6.0 * 2.0 ** e.astype(np.float64))):
        e[short] += 1
    codes = e2m1_codes(x * 2.0 ** -e[..., None].astype(np.float64))
    return codes.reshape(*codes.shape[:-2], 32 * codes.shape[-2]), np.where(bad, 128, e)


def held4_ref(codes, e):
    """What codes and exponents of quantise4_ref stand for."""
    v = E2M1[codes % 8] * np.where(codes >= 8, -1.0, 1.0)
    scale = np.where(e == 128, np.nan, 2.0 ** np.minimum(e, 127).astype(np.float64))
    return v * np.repeat(scale, 32, -1)


def page_scores_ref(q, lo, hi):
    """q [rows, d], lo, hi [pages, d] -> [pages]: the largest over the rows of the bound on q . key."""
    q = np.asarray(q, np.float64)[:, None]
    return np.where(q >= 0, q * hi, q * lo).sum(-1).max(0)


def select_ref(score, top_k, n_first, n_last):
    """Ascending indices of the top_k best pages: forced ones first, then NaN, then by score, ties to the lower."""
    n = len(score)
    key = [(0 if j < n_first or j >= n - n_last else 1 if np.isnan(score[j]) else 2,
            0.0 if np.isnan(score[j]) or j < n_first or j >= n - n_last else -score[j], j) for j in range(n)]
    return sorted(j for _, _, j in sorted(key)[:top_k])


def attn_ref(q, k, v, ends, scale, pos=None, lows=None, first=0):
    """q [rows, d], k, v [keys, d]; row r sees the keys whose position (pos, or their index) is below ends[r], and with
    lows at least lows[r] or below first.

    Returns o, lse, mass (sum of the weights times |v|, per element) and spread (the largest scale * sum |q_i k_i| of
    a visible key), which the tolerances of the tests are made of."""
    q, k, v = (np.asarray(a, np.float64) for a in (q, k, v))
    pos = np.arange(len(k)) if pos is None else np.asarray(pos)
    o, mass = np.zeros_like(q), np.zeros_like(q)
    lse, spread = np.full(len(q), -np.inf), np.zeros(len(q))
    for r in range(len(q)):
        seen = pos < ends[r]
        if lows is not None:
            seen = seen & ((pos >= lows[r]) | (pos < first))
        if not seen.any():
            continue
        s = scale * (k[seen] @ q[r])
        top = s.max()
        if top == -np.inf:
            continue
        w = np.exp(s - top)
        lse[r] = top + np.log(w.sum())
        w = w / w.sum()
        o[r] = w @ v[seen]
        mass[r] = w @ np.abs(v[seen])
        spread[r] = scale * (np.abs(k[seen]) @ np.abs(q[r])).max()
    return o, lse, mass, spread
