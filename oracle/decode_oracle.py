"""CPU oracle for the operators of token-by-token decoding.  TEST INFRASTRUCTURE ONLY.

Plain NumPy definitions, in 64 bits, of the caches' 8-bit format, attention over a cache, one step of beam search over
several beams, and the reordering of the beams' states.  Slow on purpose, shares no code with the HIP path.
"""
from __future__ import annotations

import numpy as np


def e4m3_values() -> np.ndarray:
    """The 256 values of the OCP e4m3 format by their codes (no infinities; 0x7f and 0xff are NaN)."""
    out = np.empty(256)
    for c in range(256):
        sign, e, m = -1.0 if c & 128 else 1.0, (c >> 3) & 15, c & 7
        out[c] = np.nan if e == 15 and m == 7 else sign * (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
    return out


def quantise(x: np.ndarray):
    """x [.., 64] of fp32's range -> (values q [.., 64], biased exponents [..]): e = the smallest whole number >= -127 with max|x| <= 448 2^e over
    the finite x, q = x 2^-e rounded to e4m3, ties to the even code, but to 240 where 2^128 would be nearest; NaN where x is not finite."""
    x = np.asarray(x, np.float64)
    fine = np.isfinite(x)
    largest = np.where(fine, np.abs(x), 0.0).max(-1)
    e = np.full(largest.shape, -127, np.int64)
    for i in np.ndindex(*largest.shape):
        while largest[i] > 448.0 * 2.0 ** int(e[i]):
            e[i] += 1
    y = np.where(fine, x, 0.0) * 2.0 ** (-e[..., None]).astype(np.float64)
    mag = e4m3_values()[:127]                                  # 0 .. 448 by code
    a = np.abs(y)
    hi = np.clip(np.searchsorted(mag, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = mag[hi] - a, a - mag[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = np.where(mag[hi] == a, hi, code)
    most = np.where(e[..., None] >= 120, 240.0, 448.0)         # q 2^e below 2^128
    q = np.where(fine, np.copysign(np.minimum(mag[code], most), y), np.nan)
    return q, e + 127


def cache_rows(cu, row, n_rows: int, n_tokens: int) -> np.ndarray:
    """Cache row of every token: -1 outside the cache, -2 behind the last sequence."""
    out = np.full(n_tokens, -2, np.int64)
    for s in range(len(row)):
        for t in range(cu[s], min(cu[s + 1], n_tokens)):
            r = row[s] + t - cu[s]
            out[t] = r if 0 <= r < n_rows else -1
    return out


def attention(q: np.ndarray, k: np.ndarray, v: np.ndarray, scale: float, seen: np.ndarray):
    """One row of one head: q [64], k, v [L, 64], seen [L].  Returns (out [64], the sum of w |v| [64], the largest sum of |q k| scale)."""
    k, v = np.asarray(k, np.float64)[seen], np.asarray(v, np.float64)[seen]
    if not len(k):
        return np.zeros(64), np.zeros(64), 0.0
    s = k @ np.asarray(q, np.float64) * scale
    w = np.exp(s - s.max())
    w /= w.sum()
    return w @ v, w @ np.abs(v), float((np.abs(k) @ np.abs(q) * abs(scale)).max())


def visible(n_keys: int, words=None, since: int = 0) -> np.ndarray:
    """Which keys a row sees: all of them, or those before `since` and those whose bit is set in its mask words."""
    seen = np.ones(n_keys, bool)
    if words is not None:
        for k in range(max(since, 0), n_keys):
            at = k - since
            seen[k] = at < 32 * len(words) and (int(words[at // 32]) >> (at % 32)) & 1
    return seen


def beam_step(logits, scores, n_in: int, n_out: int, done=None, eos: int = -1, keep_slots: bool = False):
    """One stream: logits [W, V], scores [W].  Returns (tokens, parents, scores in 64 bits, done) [W]."""
    W, V = np.shape(logits)
    found = []                                                  # (-total, beam, rank inside the beam, token)
    for b in range(n_in):
        if not np.isfinite(scores[b]):
            continue
        if done is not None and done[b]:
            found.append((-float(scores[b]), b, 0, eos))
            continue
        x = np.asarray(logits[b], np.float64)
        fine = np.flatnonzero(np.isfinite(x))
        if not len(fine):
            continue
        top = x[fine].max()
        lse = top + np.log(np.exp(x[fine] - top).sum())
        best = sorted(fine.tolist(), key=lambda t: (-x[t], t))[:W]
        found += [(-(float(scores[b]) + (x[t] - lse)), b, i, t) for i, t in enumerate(best)]
    found = sorted(found)[:n_out]
    slots = [None] * W
    if keep_slots:
        rest = []
        for f in found:
            if f[1] < n_out and slots[f[1]] is None:
                slots[f[1]] = f
            else:
                rest.append(f)
        for f in rest:
            slots[slots.index(None)] = f
    else:
        slots[:len(found)] = found
    tok = np.array([-1 if f is None else f[3] for f in slots])
    par = np.array([-1 if f is None else f[1] for f in slots])
    sc = np.array([-np.inf if f is None else -f[0] for f in slots])
    dn = np.array([f is not None and (f[3] == eos or bool(done is not None and done[f[1]])) for f in slots])
    return tok, par, sc, dn


def reorder(state: np.ndarray, parents: np.ndarray, lens, into: np.ndarray) -> np.ndarray:
    """state, into [layers, B * W, n_pos, ..]; parents [B, W]; lens [B].  A new array."""
    out = into.copy()
    B, W = parents.shape
    for s in range(B):
        n = min(max(int(lens[s]), 0), state.shape[2]) if lens is not None else state.shape[2]
        for j in range(W):
            if 0 <= parents[s, j] < W:
                out[:, s * W + j, :n] = state[:, s * W + parents[s, j], :n]
    return out
