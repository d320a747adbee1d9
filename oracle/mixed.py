"""Rotary positions and mixed sets that grow and are cut back, in float64 from the definitions.

rotate   pair i of the first 2 len(freqs) elements of a row at position p, as a complex number, times magnitude * e^{j p freqs[i]}
         (transpose: e^{-j p freqs[i]}); pairs are elements i and i + len(freqs), or 2 i and 2 i + 1
attend   per query b, token t and head h of KV head g, over the rows r < len[b] that the token sees:
             s = scale q.k,  x = softcap tanh(s / softcap) (or s) - slopes[h] |pq - pk|,  O = softmax(x) V,  LSE = log sum exp(x)
         sees: pq >= 0 and pk >= 0 and (pk < n_always or ((not causal or pk <= pq) and (no window or pq - pk < window)));
         the weight of a row grows by the probabilities that it receives from the tokens and heads of its KV head
evict    the n = min(len, keep) rows that come first by (protected, weight, not empty), ties to the lower row; those below n stay,
         those above fill the holes in order
"""
import math

import numpy as np


def rotate(x, positions, freqs, interleaved=False, magnitude=1.0, transpose=False):
    """x [..., N, D] at positions [N]."""
    x = np.array(x, dtype=np.float64)
    half = len(freqs)
    first, second = (np.s_[..., 0:2 * half:2], np.s_[..., 1:2 * half:2]) if interleaved else (np.s_[..., :half], np.s_[..., half:2 * half])
    angle = np.asarray(positions, np.float64)[:, None] * np.asarray(freqs, np.float64)
    z = (x[first] + 1j * x[second]) * (magnitude * np.exp((-1j if transpose else 1j) * angle))
    x[first], x[second] = z.real, z.imag
    return x


def visible(q_pos, row_pos, causal=False, window=0, n_always=0):
    """bool [T, n] of token positions [T] and row positions [n]."""
    q, k = np.asarray(q_pos, np.int64)[:, None], np.asarray(row_pos, np.int64)[None]
    by_place = np.ones(np.broadcast_shapes(q.shape, k.shape), bool)
    if causal:
        by_place &= k <= q
    if window:
        by_place &= q - k < window
    return (q >= 0) & (k >= 0) & ((k < n_always) | by_place)


def attend_mixed(qd, kmix, vmix, lens, scale=0.0, q_pos=None, row_pos=None, softcap=0.0, causal=False, window=0, n_always=0, slopes=None,
                 weight=None):
    """qd [B,T,Hq,D], kmix / vmix [B,Hkv,cap,D], q_pos [B,T], row_pos [B,Hkv,cap] -> O, LSE [B,T,Hq], weight [B,Hkv,cap] (`weight` plus
    what the rows receive; rows behind the length as given).  NaN and infinities as the formulas have them."""
    bsz, t, hq, d = qd.shape
    hkv, cap = kmix.shape[1:3]
    scale = scale or 1.0 / math.sqrt(d)
    out, lse = np.zeros((bsz, t, hq, d)), np.full((bsz, t, hq), -np.inf)
    total = np.zeros((bsz, hkv, cap)) if weight is None else np.array(weight, np.float64)
    for b in range(bsz):
        n = min(max(int(lens[b]), 0), cap)
        for h in range(hq):
            g = h // (hq // hkv)
            see = np.ones((t, n), bool) if q_pos is None else visible(q_pos[b], row_pos[b, g, :n], causal, window, n_always)
            for i in range(t):
                rows = np.flatnonzero(see[i])
                with np.errstate(all="ignore"):
                    x = kmix[b, g, rows].astype(np.float64) @ qd[b, i, h].astype(np.float64) * scale
                    if softcap:
                        x = softcap * np.tanh(x / softcap)
                    if slopes is not None:
                        x = x - float(slopes[h]) * np.abs(float(q_pos[b, i]) - row_pos[b, g, rows])
                    if not len(rows) or np.all(x == -np.inf):
                        continue
                    top = x.max()
                    p = np.exp(x - top)
                    p[x == -np.inf] = 0.0
                    if np.isnan(top) or top == np.inf:
                        p[:] = np.nan
                    used = p != 0
                    out[b, i, h] = (p[used] / p.sum()) @ vmix[b, g, rows[used]].astype(np.float64)
                    lse[b, i, h] = top + np.log(p.sum()) if not np.isnan(p).any() else np.nan
                    total[b, g, rows] += p / p.sum()
    return out, lse, total


def evict_rows(length, weight, row_pos, newest, keep, n_first=0, n_recent=0):
    """Source rows of the result of one set (int64 [n])."""
    n = min(max(int(length), 0), keep)
    length = max(int(length), 0)

    def rank(r):
        p, w = int(row_pos[r]), float(weight[r])
        if p < 0:
            return (3, 0.0, r)
        if p < n_first or (n_recent and int(newest) - p < n_recent):
            return (0, 0.0, r)
        return (2, 0.0, r) if math.isnan(w) else (1, -w, r)
    kept = sorted(sorted(range(length), key=rank)[:n])
    movers = [r for r in kept if r >= n]
    have = set(kept)
    return np.array([r if r in have else movers.pop(0) for r in range(n)], np.int64)
