"""Float64 oracle of the sequence operators, from their definitions: causal convolution, selective
scan, block norm, distillation loss, each with its backward.

Arguments are NumPy arrays as the GPU calls take them (any float type; everything is computed in
float64).  `lengths` are the sequences' numbers of tokens; what the arrays hold beyond them is not
looked at.
"""

import numpy as np


def _f64(*arrays):
    return [None if a is None else np.asarray(a, dtype=np.float64) for a in arrays]


def _count(lengths, B, L):
    return [L] * B if lengths is None else [min(max(int(n), 0), L) for n in lengths]


def sigmoid(v):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-v))


# ----------------------------------------------------------------------------
# causal convolution
# ----------------------------------------------------------------------------
def causal_conv(x, w, bias=None, silu=False, state=None, lengths=None):
    """-> (y, new_state)."""
    x, w, bias, state = _f64(x, w, bias, state)
    B, L, D = x.shape
    n = w.shape[1]
    y, new = np.zeros((B, L, D)), np.zeros((B, n - 1, D))
    for b, count in enumerate(_count(lengths, B, L)):
        seen = np.concatenate([np.zeros((n - 1, D)) if state is None else state[b], x[b, :count]])
        for t in range(count):
            p = (seen[t:t + n] * w.T).sum(0) + (0 if bias is None else bias)
            y[b, t] = p * sigmoid(p) if silu else p
        new[b] = seen[count:]
    return y, new


def causal_conv_backward(gy, x, w, bias=None, silu=False, state=None, lengths=None):
    """-> (gx, gw, gbias)."""
    gy, x, w, bias, state = _f64(gy, x, w, bias, state)
    B, L, D = x.shape
    n = w.shape[1]
    gx, gw, gbias = np.zeros((B, L, D)), np.zeros((D, n)), np.zeros(D)
    for b, count in enumerate(_count(lengths, B, L)):
        seen = np.concatenate([np.zeros((n - 1, D)) if state is None else state[b], x[b, :count]])
        for t in range(count):
            p = (seen[t:t + n] * w.T).sum(0) + (0 if bias is None else bias)
            sg = sigmoid(p)
            gp = gy[b, t] * (sg * (1 + p * (1 - sg)) if silu else 1.0)
            gw += gp[:, None] * seen[t:t + n].T
            gbias += gp
            for j in range(n):
                if t - n + 1 + j >= 0:
                    gx[b, t - n + 1 + j] += gp * w[:, j]
    return gx, gw, gbias


# ----------------------------------------------------------------------------
# selective scan
# ----------------------------------------------------------------------------
def _scan_token(x, dt, A, B, dt_bias, softplus, b, t, per):
    raw = dt[b, t] + (0 if dt_bias is None else dt_bias)
    delta = np.logaddexp(0.0, raw) if softplus else raw
    return raw, delta, np.exp(delta[:, None] * A), np.repeat(B[b, t], per, 0)


def scan(x, dt, A, B, C, skip=None, gate=None, dt_bias=None, softplus=True, h0=None, lengths=None):
    """-> (y, h_last, states [B][L + 1][D][N])."""
    x, dt, A, B, C, skip, gate, dt_bias, h0 = _f64(x, dt, A, B, C, skip, gate, dt_bias, h0)
    nb, L, D = x.shape
    N, per = A.shape[1], D // B.shape[2]
    y, states = np.zeros((nb, L, D)), np.zeros((nb, L + 1, D, N))
    last = np.zeros((nb, D, N))
    for b, count in enumerate(_count(lengths, nb, L)):
        h = np.zeros((D, N)) if h0 is None else h0[b]
        states[b, 0] = h
        for t in range(count):
            _, delta, a, Bt = _scan_token(x, dt, A, B, dt_bias, softplus, b, t, per)
            h = a * h + (delta * x[b, t])[:, None] * Bt
            states[b, t + 1] = h
            out = (h * np.repeat(C[b, t], per, 0)).sum(1) + (0 if skip is None else skip * x[b, t])
            y[b, t] = out if gate is None else out * gate[b, t] * sigmoid(gate[b, t])
        last[b] = h
    return y, last, states


def scan_backward(gy, x, dt, A, B, C, skip=None, gate=None, dt_bias=None, softplus=True, h0=None, lengths=None):
    """-> dict of the gradients of x, dt, A, B, C, skip, gate, dt_bias."""
    gy, x, dt, A, B, C, skip, gate, dt_bias, h0 = _f64(gy, x, dt, A, B, C, skip, gate, dt_bias, h0)
    _, _, states = scan(x, dt, A, B, C, skip, gate, dt_bias, softplus, h0, lengths)
    nb, L, D = x.shape
    N, G = A.shape[1], B.shape[2]
    per = D // G
    g = {"x": np.zeros_like(x), "dt": np.zeros_like(x), "A": np.zeros_like(A), "B": np.zeros(B.shape),
         "C": np.zeros(B.shape), "skip": np.zeros(D), "gate": np.zeros_like(x), "dt_bias": np.zeros(D)}
    for b, count in enumerate(_count(lengths, nb, L)):
        adj = np.zeros((D, N))
        for t in reversed(range(count)):
            raw, delta, a, Bt = _scan_token(x, dt, A, B, dt_bias, softplus, b, t, per)
            Ct, h, before = np.repeat(C[b, t], per, 0), states[b, t + 1], states[b, t]
            out = (h * Ct).sum(1) + (0 if skip is None else skip * x[b, t])
            gs = gy[b, t]
            if gate is not None:
                sg = sigmoid(gate[b, t])
                g["gate"][b, t] = gs * out * sg * (1 + gate[b, t] * (1 - sg))
                gs = gs * gate[b, t] * sg
            adj = adj + gs[:, None] * Ct
            g["C"][b, t] = (h * gs[:, None]).reshape(G, per, N).sum(1)
            g["B"][b, t] = (adj * (delta * x[b, t])[:, None]).reshape(G, per, N).sum(1)
            gu = (adj * Bt).sum(1)
            e = adj * a * before
            gdelta = (e * A).sum(1) + gu * x[b, t]
            graw = gdelta * sigmoid(raw) if softplus else gdelta
            g["x"][b, t] = gu * delta + (0 if skip is None else gs * skip)
            g["dt"][b, t] = graw
            g["A"] += e * delta[:, None]
            g["skip"] += gs * x[b, t]
            g["dt_bias"] += graw
            adj = adj * a
    return g


# ----------------------------------------------------------------------------
# block norm
# ----------------------------------------------------------------------------
_ACT = {"none": lambda g: g, "sigmoid": sigmoid, "silu": lambda g: g * sigmoid(g)}
_SLOPE = {"none": np.ones_like, "sigmoid": lambda g: sigmoid(g) * (1 - sigmoid(g)),
          "silu": lambda g: sigmoid(g) * (1 + g * (1 - sigmoid(g)))}


def _rms(v, eps):
    return 1.0 / np.sqrt((v * v).mean(1, keepdims=True) + eps)


def block_norm(x, f=None, gate=None, scale=None, w_post=None, w_pre=None, act="silu", eps=1e-6):
    """-> (out, n); n is None without w_pre."""
    x, f, gate, scale, w_post, w_pre = _f64(x, f, gate, scale, w_post, w_pre)
    out = x
    if f is not None:
        post = f if w_post is None else f * _rms(f, eps) * w_post
        out = x + (1 if scale is None else scale) * (1 if gate is None else _ACT[act](gate)) * post
    return out, None if w_pre is None else out * _rms(out, eps) * w_pre


def block_norm_backward(gout, gn, x, f=None, gate=None, scale=None, w_post=None, w_pre=None, act="silu", eps=1e-6):
    """-> dict of the gradients of what is given."""
    gout, gn, x, f, gate, scale, w_post, w_pre = _f64(gout, gn, x, f, gate, scale, w_post, w_pre)
    out, _ = block_norm(x, f, gate, scale, w_post, w_pre, act, eps)
    go = np.zeros_like(x) if gout is None else gout.copy()
    g = {}
    if w_pre is not None:
        gn = np.zeros_like(x) if gn is None else gn
        r = _rms(out, eps)
        v = gn * w_pre
        go = go + v * r - out * r ** 3 * (v * out).mean(1, keepdims=True)
        g["w_pre"] = (gn * out * r).sum(0)
    g["x"] = go
    if f is None:
        return g
    rf = _rms(f, eps)
    post = f if w_post is None else f * rf * w_post
    a = np.ones_like(x) if gate is None else _ACT[act](gate)
    s = np.ones(x.shape[1]) if scale is None else scale
    if scale is not None:
        g["scale"] = (go * a * post).sum(0)
    if gate is not None:
        g["gate"] = go * s * post * _SLOPE[act](gate)
    gpost = go * s * a
    if w_post is None:
        g["f"] = gpost
    else:
        g["w_post"] = (gpost * f * rf).sum(0)
        u = gpost * w_post
        g["f"] = u * rf - f * rf ** 3 * (u * f).mean(1, keepdims=True)
    return g


# ----------------------------------------------------------------------------
# distillation
# ----------------------------------------------------------------------------
def _log_softmax(v):
    """From the differences to the largest value: m + log(sum) would lose the logarithm next to an m of 1e38."""
    d = v - v.max()
    return d - np.log(np.exp(d).sum())


def distill(z, idx, teacher, temperature=1.0, labels=None, alpha=1.0, weight=None, gloss=None):
    """-> (loss [rows], gz): the gradient for gloss [rows] (ones if None)."""
    z, teacher, weight, gloss = _f64(z, teacher, weight, gloss)
    R, V = z.shape
    loss, gz = np.zeros(R), np.zeros((R, V))
    for r in range(R):
        w = 1.0 if weight is None else weight[r]
        if w == 0:
            continue
        label = -1 if labels is None else int(labels[r])
        if label >= V or (idx[r] >= V).any():
            loss[r], gz[r] = np.nan, np.nan
            continue
        g = w * (1.0 if gloss is None else gloss[r])
        if label >= 0:
            lp = _log_softmax(z[r])
            loss[r] -= w * (1 - alpha) * lp[label]
            gz[r] += g * (1 - alpha) * np.exp(lp)
            gz[r, label] -= g * (1 - alpha)
        at = np.flatnonzero(idx[r] >= 0)
        t = teacher[r, at] / temperature
        if len(at) == 0 or np.all(t == -np.inf):
            continue
        lp = _log_softmax(z[r] / temperature)
        lq = _log_softmax(t)
        q = np.exp(lq)
        on = q > 0
        kl = q[on] * (lq[on] - lp[idx[r, at][on]])
        loss[r] += w * alpha * temperature ** 2 * kl.sum()
        gz[r] += g * alpha * temperature * np.exp(lp)
        np.subtract.at(gz[r], idx[r, at], g * alpha * temperature * q)
    return loss, gz
