"""Plain 64-bit statements of tree attention, the 8-bit cache format and token log probabilities, for the tests. numpy
only; nothing here is shared with the library."""
import math

import numpy as np


def e4m3_values() -> np.ndarray:
    """Sign, 4 bits of exponent (bias 7), 3 of mantissa; 0x7f and 0xff are no numbers."""
    v = np.empty(256)
    for b in range(256):
        e, m = b >> 3 & 15, b & 7
        x = math.nan if (e, m) == (15, 7) else (1 + m / 8) * 2.0 ** (e - 7) if e else m / 8 * 2.0 ** -6
        v[b] = -x if b >> 7 else x
    return v


E4M3 = e4m3_values()
_CODES = np.arange(0x7F)                                        # the finite magnitudes in ascending order


def quantise_row(x: np.ndarray):
    """(codes uint8, scale byte) of one row of float64 values: nearest code, ties to the even one. A row with a NaN: byte 255."""
    if np.isnan(x).any():
        return np.where(np.isnan(x), 0x7F, 0).astype(np.uint8), 255
    most = np.abs(x).max()
    if most == 0:
        E = 0
    elif np.isinf(most):
        E = 62
    else:
        E = -200
        while most > 448 * 2.0 ** E:
            E += 1
        E = min(max(E, -62), 62)
    mags = E4M3[_CODES]
    codes = np.empty(len(x), np.uint8)
    for i, v in enumerate(x):
        a = min(abs(v) * 2.0 ** -E, 448.0)
        hi = int(np.searchsorted(mags, a))
        lo = max(hi - 1, 0)
        hi = min(hi, len(mags) - 1)
        d_lo, d_hi = a - mags[lo], mags[hi] - a
        c = lo if d_lo < d_hi else hi if d_hi < d_lo else (lo if lo % 2 == 0 else hi)
        codes[i] = c | (0x80 if np.signbit(v) else 0)
    return codes, E + 127


def attention(q, k, v, seen, scale):
    """q [t, hq, d], k and v [n, hkv, d] float64, seen [t, n] bool -> (out [t, hq, d], sum p|v|): keys that are not seen do
    not take part whatever they hold; a query that sees none gets zeros."""
    t, hq, d = q.shape
    g = hq // k.shape[1]
    out, bound = np.zeros((t, hq, d)), np.zeros((t, hq, d))
    for i in range(t):
        keys = np.flatnonzero(seen[i])
        if len(keys) == 0:
            continue
        for h in range(hq):
            s = k[keys, h // g] @ q[i, h] * scale
            p = np.exp(s - s.max())
            p /= p.sum()
            out[i, h] = p @ v[keys, h // g]
            bound[i, h] = p @ np.abs(v[keys, h // g])
    return out, bound


def token_logprobs(x, scale, tokens, n_top):
    """One row of float64 logits -> (logprob, rank, entropy, top_logprob, top_token)."""
    y = x * scale
    bad = np.isnan(x).any() or np.isposinf(x).any()
    real = np.flatnonzero(~np.isnan(x))
    order = real[np.argsort(-x[real], kind="stable")]          # descending, equal ones by index
    place = {int(t): i for i, t in enumerate(order)}
    if bad:
        lp, ent = np.full(len(x), np.nan), np.nan
    elif not np.isfinite(x).any():
        lp, ent = np.full(len(x), -np.inf), 0.0
    else:
        m = y.max()
        z = np.exp(y - m).sum()
        lp = y - m - np.log(z)
        p = np.exp(lp)
        ent = -(p[p > 0] * lp[p > 0]).sum()
    logprob = [lp[t] if 0 <= t < len(x) and not np.isnan(x[t]) else np.nan for t in tokens]
    rank = [place[t] if 0 <= t < len(x) and t in place else -1 for t in tokens]
    top = [int(t) for t in order[:n_top]] + [-1] * max(0, n_top - len(order))
    top_lp = [lp[t] if t >= 0 else np.nan for t in top]
    return np.array(logprob), np.array(rank), ent, np.array(top_lp), np.array(top)
