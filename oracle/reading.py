"""Float64 oracle of the operators that read an image's tokens and score answers, from their definitions:
rotary positions of several axes, cross attention, token log probabilities, each with its backward.

Arguments are NumPy arrays as the GPU calls take them (any float type; everything is computed in float64).
What the arrays hold past a sequence's lengths, or at keys that a mask hides, is not looked at.
"""

import numpy as np

from .sequence import _count, _f64


# ----------------------------------------------------------------------------
# rotary positions
# ----------------------------------------------------------------------------
def rotary(x, positions, freqs, sections=None, interleaved=False, lengths=None, inverse=False):
    """x [B][L][H][D], positions [B][L][axes] (or [L][axes]) -> y.  The backward is the inverse."""
    x, freqs = _f64(x, freqs)
    B, L, H, D = x.shape
    positions = np.broadcast_to(np.asarray(positions), (B, L, np.shape(positions)[-1])).astype(np.float64)
    sections = (len(freqs),) if sections is None else sections
    P = len(freqs)
    y = np.zeros((B, L, H, D))
    for b, count in enumerate(_count(lengths, B, L)):
        y[b, :count] = x[b, :count]
        pair = 0
        for axis, n in enumerate(sections):
            for _ in range(n):
                a = positions[b, :count, axis] * freqs[pair] * (-1 if inverse else 1)
                i, j = (2 * pair, 2 * pair + 1) if interleaved else (pair, P + pair)
                u, v = x[b, :count, :, i], x[b, :count, :, j]
                c, s = np.cos(a)[:, None], np.sin(a)[:, None]
                y[b, :count, :, i], y[b, :count, :, j] = u * c - v * s, u * s + v * c
                pair += 1
    return y


# ----------------------------------------------------------------------------
# cross attention
# ----------------------------------------------------------------------------
def _keys(b, Lk, lengths, mask):
    there = np.ones(Lk, dtype=bool) if mask is None else np.asarray(mask)[b].astype(bool)
    if lengths is not None:
        there = there & (np.arange(Lk) < int(np.asarray(lengths)[b]))
    return np.nonzero(there)[0]


def _softmax_rows(s):
    """Softmax and log sum exp of each row."""
    with np.errstate(invalid="ignore"):
        m = s.max(1, keepdims=True)
        e = np.exp(s - m)
    total = e.sum(1, keepdims=True)
    return e / total, (m + np.log(total))[:, 0]


def cross_attention(q, k, v, scale=None, q_lengths=None, lengths=None, mask=None):
    """-> (y [B][Lq][H][D], lse [B][H][Lq])."""
    q, k, v = _f64(q, k, v)
    B, Lq, H, D = q.shape
    Lk, G = k.shape[1:3]
    scale = D ** -0.5 if scale is None else scale
    y, lse = np.zeros((B, Lq, H, D)), np.full((B, H, Lq), -np.inf)
    for b, n in enumerate(_count(q_lengths, B, Lq)):
        at = _keys(b, Lk, lengths, mask)
        if not len(at) or not n:
            continue
        for h in range(H):
            g = h // (H // G)
            p, lse[b, h, :n] = _softmax_rows(q[b, :n, h] @ k[b, at, g].T * scale)
            y[b, :n, h] = p @ v[b, at, g]
    return y, lse


def cross_attention_backward(gy, q, k, v, scale=None, q_lengths=None, lengths=None, mask=None):
    """-> (gq, gk, gv)."""
    gy, q, k, v = _f64(gy, q, k, v)
    B, Lq, H, D = q.shape
    Lk, G = k.shape[1:3]
    scale = D ** -0.5 if scale is None else scale
    gq, gk, gv = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    for b, n in enumerate(_count(q_lengths, B, Lq)):
        at = _keys(b, Lk, lengths, mask)
        if not len(at) or not n:
            continue
        for h in range(H):
            g = h // (H // G)
            p, _ = _softmax_rows(q[b, :n, h] @ k[b, at, g].T * scale)
            gp = gy[b, :n, h] @ v[b, at, g].T
            gs = p * (gp - (p * gp).sum(1, keepdims=True)) * scale
            gq[b, :n, h] = gs @ k[b, at, g]
            gk[b, at, g] += gs.T @ q[b, :n, h]
            gv[b, at, g] += p.T @ gy[b, :n, h]
    return gq, gk, gv


# ----------------------------------------------------------------------------
# token log probabilities
# ----------------------------------------------------------------------------
def best(row, K):
    """The places of the K largest of a row, from high to low, equal ones by place; a NaN counts as the largest."""
    key = np.where(np.isnan(row), np.inf, row)
    order = np.lexsort((np.arange(len(row)), -key, ~np.isnan(row)))
    return order[:K]


def _log_softmax(row, temperature):
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        d = (row - row.max()) / temperature
        return d - np.log(np.exp(d).sum())


def token_logprobs(z, tokens=None, top=0, temperature=1.0):
    """-> (logp [R], entropy [R], idx [R][top], values [R][top]); logp is None without tokens."""
    (z,) = _f64(z)
    R, V = z.shape
    logp = None if tokens is None else np.zeros(R)
    entropy, idx, values = np.zeros(R), np.zeros((R, top), dtype=np.int64), np.zeros((R, top))
    for r in range(R):
        l = _log_softmax(z[r], temperature)
        p = np.exp(l)
        entropy[r] = -np.where(p == 0, 0.0, p * np.where(p == 0, 0.0, l)).sum()
        if tokens is not None and tokens[r] >= 0:
            logp[r] = l[tokens[r]] if tokens[r] < V else np.nan
        idx[r] = best(z[r], top)
        values[r] = l[idx[r]]
    return logp, entropy, idx, values


def token_logprobs_backward(z, tokens=None, glogp=None, gentropy=None, idx=None, gtop=None, temperature=1.0):
    """-> gz [R][V]."""
    z, glogp, gentropy, gtop = _f64(z, glogp, gentropy, gtop)
    R, V = z.shape
    gz = np.zeros((R, V))
    for r in range(R):
        named = [] if glogp is None or tokens[r] < 0 else [(int(tokens[r]), glogp[r])]
        if gtop is not None:
            named += [(int(v), g) for v, g in zip(idx[r], gtop[r]) if v >= 0]
        gh = 0.0 if gentropy is None else gentropy[r]
        if gh == 0 and all(g == 0 for _, g in named):
            continue
        l = _log_softmax(z[r], temperature)
        p = np.exp(l)
        entropy = -np.where(p == 0, 0.0, p * np.where(p == 0, 0.0, l)).sum()
        gl = -p * sum(g for _, g in named) - gh * np.where(p == 0, 0.0, p * (np.where(p == 0, 0.0, l) + entropy))
        for v, g in named:
            if v < V:
                gl[v] += g
            else:
                gl[:] = np.nan
        gz[r] = gl / temperature
    return gz
