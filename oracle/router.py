"""The router's operators in numpy, in 64 bits: chosen or replayed experts and
their gates, demand counts, the balance loss, and the gradient of gates and
loss.  Written from the formulas of include/routepack/router.h; shares no code
with the library.

Logits are float64 [T][L][E], ids int64 [T][L][k] (outside [0, E): no choice),
offsets int64 [N + 1].  Beside a value stands its magnitude: the sum of the
absolute terms that it is formed from, to which rounding errors are relative.
"""
from __future__ import annotations

import numpy as np


def _sigmoid(z):
    e = np.exp(-np.abs(z))
    return np.where(z >= 0, 1.0, e) / (1.0 + e), np.where(z >= 0, e, 1.0) / (1.0 + e)


def _ratio(a, b):
    return np.divide(a, b, out=np.zeros(np.broadcast_shapes(a.shape, b.shape)), where=b != 0)


def _softmax(z):
    m = z.max(axis=-1, keepdims=True, initial=-np.inf)
    e = np.exp(z - np.where(np.isneginf(m), 0.0, m))
    return _ratio(e, e.sum(axis=-1, keepdims=True))


def shares(z, score):
    """Scores divided by their sum (0 without an available expert)."""
    if score == "softmax":
        return _softmax(z)
    s, _ = _sigmoid(z)
    m = z.max(axis=-1, keepdims=True)
    low = (m < 0.0) & np.isfinite(m)  # the scores times e^-m, which stay in range
    s = np.where(low, np.exp(np.minimum(z - np.where(low, m, 0.0), 0.0)) / (1.0 + np.exp(np.minimum(z, 0.0))), s)
    return _ratio(s, s.sum(axis=-1, keepdims=True))


def choose(z, k, bias=None, score="softmax"):
    if bias is not None and score == "softmax":
        # a NaN takes no part, and experts of +inf share the scores alone
        key = _softmax(np.where(np.isnan(z), -np.inf, np.where((z == np.inf).any(axis=-1, keepdims=True),
                                                               np.where(z == np.inf, 0.0, -np.inf), z))) + bias
    else:
        key = z if bias is None else _sigmoid(z)[0] + bias
    key = np.where(np.isneginf(z) | np.isnan(z) | np.isnan(key), -np.inf, key)
    ids = np.argsort(-key, axis=-1, kind="stable")[..., :k]
    return np.where(np.isneginf(np.take_along_axis(key, ids, -1)), -1, ids)


def _chosen(z, ids, score, normalize):
    E = z.shape[-1]
    on = (ids >= 0) & (ids < E)
    at = np.where(on, ids, 0)
    zc = np.take_along_axis(z, at, -1)
    if score == "softmax" and not normalize:
        w = np.where(on, np.take_along_axis(_softmax(z), at, -1), 0.0)
    elif score == "softmax":
        w = _softmax(np.where(on, zc, -np.inf))
    elif normalize:
        w = shares(np.where(on, zc, -np.inf), "sigmoid")
    else:
        w = np.where(on, _sigmoid(zc)[0], 0.0)
    return on, at, zc, w


def gates(z, ids, score, normalize, scale):
    return scale * _chosen(z, ids, score, normalize)[3]


def count(ids, offsets, E):
    N, L = len(offsets) - 1, ids.shape[1]
    out = np.zeros((N, L, E), dtype=np.int32)
    for i in range(N):
        for l in range(L):
            x = ids[offsets[i]:offsets[i + 1], l].reshape(-1).astype(np.int64)
            out[i, l] = np.bincount(x[(x >= 0) & (x < E)], minlength=E)
    return out


def fractions(counts):
    c = counts.astype(np.float64)
    return _ratio(c.shape[-1] * c, c.sum(axis=-1, keepdims=True))


def balance(z, counts, offsets, score):
    """(loss [L], shares [G][L][E])."""
    G = len(offsets) - 1
    out = np.zeros(counts.shape)
    for g in range(G):
        if offsets[g + 1] > offsets[g]:
            out[g] = shares(z[offsets[g]:offsets[g + 1]], score).mean(axis=0)
    return (fractions(counts) * out).sum(axis=-1).sum(axis=0) / G, out


def backward(z, score, ids=None, dgates=None, normalize=True, scale=1.0, counts=None, offsets=None, dloss=None):
    """(dlogits, magnitude)."""
    dz, mag = np.zeros(z.shape), np.zeros(z.shape)
    p = shares(z, score)
    less = _sigmoid(z)[1]
    if ids is not None:
        on, at, zc, w = _chosen(z, ids, score, normalize)
        dg = np.where(on, dgates, 0.0)
        dot = (w * dg).sum(axis=-1, keepdims=True) if normalize else 0.0
        adot = (w * abs(dg)).sum(axis=-1, keepdims=True) if normalize else 0.0
        d, a = scale * w * (dg - dot), abs(scale) * w * (abs(dg) + adot)
        if score == "sigmoid":
            lc = np.where(on, _sigmoid(zc)[1], 0.0)
            d, a = d * lc, a * lc
        T, L, k = ids.shape
        ti, li = np.arange(T)[:, None, None], np.arange(L)[None, :, None]
        np.add.at(dz, (ti, li, at), np.where(on, d, 0.0))
        np.add.at(mag, (ti, li, at), np.where(on, a, 0.0))
        if score == "softmax" and not normalize:
            dz -= p * d.sum(axis=-1, keepdims=True)
            mag += p * a.sum(axis=-1, keepdims=True)
    if dloss is not None:
        G, f = len(offsets) - 1, fractions(counts)
        for g in range(G):
            b, e = offsets[g], offsets[g + 1]
            if e <= b:
                continue
            c = f[g] * (dloss[:, None] / (G * (e - b)))
            q = p[b:e]
            d = q * (c - (q * c).sum(axis=-1, keepdims=True))
            a = q * (abs(c) + (q * abs(c)).sum(axis=-1, keepdims=True))
            dz[b:e] += d * less[b:e] if score == "sigmoid" else d
            mag[b:e] += a * less[b:e] if score == "sigmoid" else a
    return dz, mag
