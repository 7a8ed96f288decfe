"""Plain 64-bit references (CPU, numpy) of the delta rule over packed sequences, its
gradient, and the norm and rotation of queries and keys, written from the recurrences
token by token."""
from __future__ import annotations

import numpy as np


def bounds(lengths):
    return np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)


def forward(lengths, q, k, v, la, beta, scale, s0=None):
    """o [total][HV][dv], final states [N][HV][dv][dk] and what the adjoint needs."""
    HK, dk = q.shape[1:]
    HV, dv = v.shape[1:]
    G, off = HV // HK, bounds(lengths)
    o = np.zeros((q.shape[0], HV, dv))
    last = np.zeros((len(lengths), HV, dv, dk))
    old, err = np.zeros((q.shape[0], HV, dv, dk)), np.zeros((q.shape[0], HV, dv))
    with np.errstate(divide="ignore"):
        alpha = np.exp(la)
    for n in range(len(lengths)):
        S = np.zeros((HV, dv, dk)) if s0 is None else s0[n].astype(np.float64).copy()
        for t in range(off[n], off[n + 1]):
            kt, qt = np.repeat(k[t], G, 0), np.repeat(q[t], G, 0)
            S = alpha[t][:, None, None] * S
            e = v[t] - np.einsum("hvk,hk->hv", S, kt)
            old[t], err[t] = S, e
            S = S + (beta[t][:, None] * e)[..., None] * kt[:, None, :]
            o[t] = scale * np.einsum("hvk,hk->hv", S, qt)
        last[n] = S
    return o, last, (alpha, old, err)


def backward(lengths, q, k, v, la, beta, scale, s0, do, ds):
    """Gradients by q, k, v, log_alpha, beta and the initial states."""
    HK, HV = q.shape[1], v.shape[1]
    G, off = HV // HK, bounds(lengths)
    _, last, (alpha, old, err) = forward(lengths, q, k, v, la, beta, scale, s0)
    dq, dk, dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    dla, db = np.zeros_like(la), np.zeros_like(beta)
    ds0 = np.zeros_like(last)
    for n in range(len(lengths)):
        D = np.zeros_like(last[n]) if ds is None else ds[n].astype(np.float64).copy()
        for t in range(off[n + 1] - 1, off[n] - 1, -1):
            kt, qt = np.repeat(k[t], G, 0), np.repeat(q[t], G, 0)
            be = beta[t][:, None] * err[t]
            S = old[t] + be[..., None] * kt[:, None, :]
            dqt = scale * np.einsum("hv,hvk->hk", do[t], S)
            D = D + scale * do[t][..., None] * qt[:, None, :]
            u = np.einsum("hvk,hk->hv", D, kt)
            db[t] = np.sum(u * err[t], -1)
            dv[t] = beta[t][:, None] * u
            dkt = np.einsum("hvk,hv->hk", D, be) - np.einsum("hvk,hv->hk", old[t], dv[t])
            D = D - dv[t][..., None] * kt[:, None, :]
            dla[t] = np.sum(D * old[t], (-1, -2))
            D = alpha[t][:, None, None] * D
            dq[t] = dqt.reshape(HK, G, -1).sum(1)
            dk[t] = dkt.reshape(HK, G, -1).sum(1)
        ds0[n] = D
    return dq, dk, dv, dla, db, ds0


def _turned(y, cs, rot, pairs, sign):
    if not rot:
        return y
    c, s = cs[:, None, :rot // 2], sign * cs[:, None, rot // 2:]
    z = y.copy()
    a, b = (y[..., 0:rot:2], y[..., 1:rot:2]) if pairs else (y[..., :rot // 2],
                                                             y[..., rot // 2:rot])
    x, w = a * c - b * s, b * c + a * s
    if pairs:
        z[..., 0:rot:2], z[..., 1:rot:2] = x, w
    else:
        z[..., :rot // 2], z[..., rot // 2:rot] = x, w
    return z


def norm(x, w, rms, eps, rot=0, cs=None, pairs=False):
    """x [T][H][D] normed by w (or 1), then turned by the tokens' rows of the table."""
    n = x.shape[-1] if rms else 1
    r = 1.0 / np.sqrt((x * x).sum(-1, keepdims=True) / n + eps)
    y = x * r * (1.0 if w is None else w)
    return _turned(y, cs, rot, pairs, 1.0)


def norm_backward(x, w, dz, rms, eps, rot=0, cs=None, pairs=False):
    n = x.shape[-1] if rms else 1
    r = 1.0 / np.sqrt((x * x).sum(-1, keepdims=True) / n + eps)
    dy = _turned(dz, cs, rot, pairs, -1.0)
    wd = dy * (1.0 if w is None else w)
    dx = r * (wd - x * r * r * (wd * x).sum(-1, keepdims=True) / n)
    return dx, (dy * x * r).sum((0, 1))
