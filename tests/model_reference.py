"""Plain 64-bit references (CPU, numpy) of the short causal convolution, the norms around a
block and the log probabilities of tokens, each with the size of the terms that its results
are sums of (what roundings are relative to)."""
from __future__ import annotations

import numpy as np


def sigmoid(x):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-x))


# ---- short causal convolution ---------------------------------------------------------------

def conv(lengths, x, w, bias, state, silu):
    """y, last states, and the terms' size of every sum; w [C][taps], state [N][taps - 1][C]."""
    K, C = w.shape[1], x.shape[1]
    y, size = np.zeros_like(x), np.zeros_like(x)
    last, t = np.zeros((len(lengths), K - 1, C)), 0
    for n, length in enumerate(lengths):
        rows = np.zeros((K - 1 + length, C))
        if state is not None:
            rows[:K - 1] = state[n]
        rows[K - 1:] = x[t:t + length]
        for i in range(length):
            pre = (rows[i:i + K] * w.T).sum(0) + bias
            size[t + i] = (np.abs(rows[i:i + K] * w.T)).sum(0) + np.abs(bias)
            y[t + i] = pre * sigmoid(pre) if silu else pre
        last[n] = rows[length:]
        t += length
    return y, last, size


def conv_backward(lengths, x, w, bias, state, silu, dy, dlast):
    """dx, dw, dbias, dstate and the terms' sizes of each."""
    K, C = w.shape[1], x.shape[1]
    out = [np.zeros_like(x), np.zeros_like(w), np.zeros(C), np.zeros((len(lengths), K - 1, C))]
    sizes = [np.zeros_like(o) for o in out]
    t = 0
    for n, length in enumerate(lengths):
        rows, drows = np.zeros((K - 1 + length, C)), np.zeros((K - 1 + length, C))
        if state is not None:
            rows[:K - 1] = state[n]
        rows[K - 1:] = x[t:t + length]
        dsize = np.zeros_like(drows)
        for i in range(length):
            terms = rows[i:i + K] * w.T
            pre, g, more = terms.sum(0) + bias, dy[t + i], 1.0
            if silu:
                s = sigmoid(pre)
                g = g * s * (1 + pre * (1 - s))
                more = 1.0 + np.abs(terms).sum(0) + np.abs(bias)
            gsize = np.abs(dy[t + i]) * more
            drows[i:i + K] += g * w.T
            dsize[i:i + K] += gsize * np.abs(w.T)
            out[1] += (g * rows[i:i + K]).T
            sizes[1] += (gsize * np.abs(rows[i:i + K])).T
            out[2] += g
            sizes[2] += gsize
        if dlast is not None:
            drows[length:] += dlast[n]
            dsize[length:] += np.abs(dlast[n])
        out[0][t:t + length], sizes[0][t:t + length] = drows[K - 1:], dsize[K - 1:]
        out[3][n], sizes[3][n] = drows[:K - 1], dsize[:K - 1]
        t += length
    return out, sizes


# ---- norms around a block -------------------------------------------------------------------

def _act(kind, g):
    s = sigmoid(g)
    if kind == "silu":
        return g * s, s * (1 + g * (1 - s))
    return s, s * (1 - s)


def block_norm(x, res, gate, wa, wb, cs, *, after, before, act, scale, eps):
    """(y, h) and the sizes of their terms; rows are the last axis."""
    D = x.shape[-1]
    one = np.ones(D)
    wa, wb, cs = (one if w is None else w for w in (wa, wb, cs))
    n = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) if after else x
    u = n * wa
    if act:
        u = u * _act(act, gate)[0]
    h, size = scale * cs * u, np.abs(scale * cs * u)
    if res is not None:
        h, size = h + res, size + np.abs(res)
    y, ysize = h, size
    if before:
        r = 1 / np.sqrt((h * h).mean(-1, keepdims=True) + eps)
        y, ysize = h * r * wb, size * r * np.abs(wb)
    return y, h, ysize, size


def block_norm_backward(x, res, gate, wa, wb, cs, dy, dh, *, after, before, act, scale, eps):
    """Gradients by (x, res, gate, wa, wb, cs) and the sizes of their terms."""
    D, axes = x.shape[-1], tuple(range(x.ndim - 1))
    one = np.ones(D)
    wa, wb, cs = (one if w is None else w for w in (wa, wb, cs))
    rx = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps) if after else 1.0
    n = x * rx
    a, da = _act(act, gate) if act else (1.0, 0.0)
    u = n * wa * a
    h = scale * cs * u + (0 if res is None else res)
    # the norm's mean of h and the gate's slope take h and g with their roundings
    hs = np.abs(scale * cs * u) + (0 if res is None else np.abs(res))
    d = np.zeros_like(x) if dh is None else dh.copy()
    ds = np.abs(d)
    dy = np.zeros_like(x) if dy is None else dy
    dwb = dwbs = None
    if before:
        r = 1 / np.sqrt((h * h).mean(-1, keepdims=True) + eps)
        dwb, dwbs = (dy * h * r).sum(axes), (np.abs(dy) * hs * r).sum(axes)
        d = d + r * (wb * dy - h * r * r * (wb * dy * h).mean(-1, keepdims=True))
        ds = ds + r * (np.abs(wb * dy) + hs * r * r * (np.abs(wb * dy) * hs).mean(-1, keepdims=True))
    else:
        d, ds = d + dy, ds + np.abs(dy)
    dres, dress = d, ds
    dcs, dcss = scale * (d * u).sum(axes), abs(scale) * (ds * np.abs(u)).sum(axes)
    du, dus = scale * cs * d, np.abs(scale * cs) * ds
    dg, dgs = du * n * wa * da, dus * np.abs(n * wa)
    du, dus = du * a, dus * np.abs(a)
    dwa, dwas = (du * n).sum(axes), (dus * np.abs(n)).sum(axes)
    if after:
        dx = rx * (wa * du - x * rx * rx * (wa * du * x).mean(-1, keepdims=True))
        dxs = rx * (np.abs(wa) * dus +
                    np.abs(x) * rx * rx * (np.abs(wa) * dus * np.abs(x)).mean(-1, keepdims=True))
    else:
        dx, dxs = du * wa, dus * np.abs(wa)
    return (dx, dres, dg, dwa, dwb, dcs), (dxs, dress, dgs, dwas, dwbs, dcss)


# ---- log probabilities of tokens ----------------------------------------------------------

def logprobs(x, given, K, scale):
    """(logp of given, lse, entropy, top tokens, their logp); rows of -inf alone by the rule."""
    R, V = x.shape
    lse, entropy = np.empty(R), np.empty(R)
    logp = np.empty((R, 0 if given is None else given.shape[1]))
    top, top_logp = np.empty((R, K), np.int64), np.empty((R, K))
    for r in range(R):
        row = x[r]
        with np.errstate(all="ignore"):
            if np.isneginf(row).all():
                lse[r], entropy[r], p = -np.inf, 0.0, np.full(V, -np.inf)
            elif np.isnan(row).any() or np.isposinf(row).any():
                lse[r] = entropy[r] = np.nan
                p = np.full(V, np.nan)
            else:
                m = row.max()
                d = scale * (row - m)
                s = np.exp(d).sum()
                lse[r], p = scale * m + np.log(s), d - np.log(s)
                q = np.exp(p)
                entropy[r] = -(q[q > 0] * p[q > 0]).sum()
        for g in range(logp.shape[1]):
            v = given[r, g]
            logp[r, g] = 0.0 if v < 0 else np.nan if v >= V else p[v]
        order = sorted(range(V), key=lambda v: (np.isnan(row[v]), -row[v] if row[v] == row[v] else 0,
                                                v))
        top[r] = order[:K]
        top_logp[r] = p[top[r]]
    return logp, lse, entropy, top, top_logp


def logprobs_backward(x, given, dlogp, dlse, dentropy, scale):
    """The gradient by x and the size of its terms."""
    R, V = x.shape
    out, size = np.zeros((R, V)), np.zeros((R, V))
    for r in range(R):
        if np.isneginf(x[r]).all():
            continue
        with np.errstate(all="ignore"):
            z = scale * x[r]
            m = z.max()
            l = z - m - np.log(np.exp(z - m).sum())
            p = np.exp(l)
            lz = np.where(p > 0, l, 0.0)
            H = -(p * lz).sum()
        a, asize = 0.0, 0.0
        if dlse is not None:
            a, asize = a + dlse[r], asize + abs(dlse[r])
        for g in range(0 if given is None else given.shape[1]):
            v = given[r, g]
            if v < 0:
                continue
            if v >= V:
                a = np.nan
                continue
            a, asize = a - dlogp[r, g], asize + abs(dlogp[r, g])
            out[r, v] += dlogp[r, g]
            size[r, v] += abs(dlogp[r, g])
        f, fs = np.full(V, a), np.full(V, asize)
        if dentropy is not None:
            f = f - dentropy[r] * (lz + H)
            fs = fs + abs(dentropy[r]) * (np.abs(lz) + H)
        out[r] += p * f
        size[r] += p * fs
    return scale * out, scale * size
