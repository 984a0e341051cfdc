"""The experts' operators in numpy, in 64 bits: choices among groups of experts,
the order of pairs by slot, matrices in microscaled 4-bit floating point, the
experts' products and sums with their gradients.  Written from the formulas of
include/routepack/router.h and experts.h; shares no code with the library."""
from __future__ import annotations

import numpy as np

from . import router

STEPS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def choose_groups(z, k, groups, keep, top=1, bias=None, score="softmax"):
    """int64 [T][L][k]: -1 where no available expert is left."""
    T, L, E = z.shape
    zero = np.zeros((L, E)) if bias is None else bias
    if bias is None and top == 1:
        key = z
    elif score == "softmax":
        # a NaN takes no part, and experts of +inf share the scores alone
        inf = (z == np.inf).any(axis=-1, keepdims=True)
        key = router._softmax(np.where(np.isnan(z), -np.inf, np.where(inf, np.where(z == np.inf, 0.0, -np.inf), z))) + zero
    else:
        key = router._sigmoid(z)[0] + zero
    key = np.where(np.isneginf(z) | np.isnan(z) | np.isnan(key), -np.inf, key)
    by = -np.sort(-key.reshape(T, L, groups, E // groups), axis=-1)[..., :top]
    best = np.where(np.isneginf(by[..., 0]), -np.inf, np.where(np.isneginf(by), 0.0, by).sum(axis=-1))
    first = np.argsort(-best, axis=-1, kind="stable")[..., :keep]
    on = np.zeros((T, L, groups), dtype=bool)
    np.put_along_axis(on, first, True, axis=-1)
    on &= ~np.isneginf(best)
    key = np.where(np.repeat(on, E // groups, axis=-1), key, -np.inf)
    ids = np.argsort(-key, axis=-1, kind="stable")[..., :k]
    return np.where(np.isneginf(np.take_along_axis(key, ids, -1)), -1, ids)


def order(ids, E, slots=None):
    """(rows [L][T k], offsets [L][E + 1], places [T][L][k])."""
    T, L, k = ids.shape
    rows = np.full((L, T * k), -1, dtype=np.int64)
    offsets = np.zeros((L, E + 1), dtype=np.int64)
    places = np.full((T, L, k), -1, dtype=np.int64)
    for l in range(L):
        by = [[] for _ in range(E)]
        for t in range(T):
            for j in range(k):
                e = ids[t, l, j]
                if 0 <= e < E:
                    s = e if slots is None else slots[l, e]
                    if 0 <= s < E:
                        by[s].append((t, j))
        r = 0
        for s in range(E):
            for t, j in by[s]:
                rows[l, r], places[t, l, j] = t * k + j, r
                r += 1
            offsets[l, s + 1] = r
    return rows, offsets, places


def quantize(x):
    """(codes uint8 [R][64 n], scales uint8 [R][4 n]) of x [R][C], n = ceil(C / 128)."""
    R, C = x.shape
    v = np.zeros((R, (C + 127) // 128 * 128))
    v[:, :C] = x
    b = v.reshape(R, -1, 32)
    odd = ~np.isfinite(b).all(axis=2)
    b = np.where(odd[..., None], 0.0, b)
    big = np.abs(b).max(axis=2)
    e = np.where(big > 0, np.frexp(big)[1] - 3, -127).clip(-127)
    m = np.abs(b) * 2.0 ** -e[..., None]
    # the nearest step, of two as near the one with an even code
    d = np.abs(m[..., None] - STEPS)
    near = np.where(d == d.min(axis=-1, keepdims=True), np.arange(8) % 2, 2)
    code = np.where(m >= 6.0, 7, np.argmin(near, axis=-1))
    code = code + 8 * np.signbit(b)
    code = np.where(odd[..., None], 0, code).reshape(R, -1, 2)
    return (code[..., 0] + 16 * code[..., 1]).astype(np.uint8), np.where(odd, 255, e + 127).astype(np.uint8)


def values(codes, scales, C):
    """The values of a matrix in 4 bits, float64 [...][C]."""
    c = np.stack((codes & 15, codes >> 4), axis=-1).reshape(*codes.shape[:-1], -1)
    v = np.where(c >= 8, -1.0, 1.0) * STEPS[c & 7]
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127.0))
    return (v.reshape(*scales.shape, 32) * s[..., None]).reshape(*codes.shape[:-1], -1)[..., :C]


def product(x, w, offsets):
    """(y, magnitude) of rows x [P][C] by the matrices w [E][N][C]."""
    y, mag = (np.zeros((x.shape[0], w.shape[1])) for _ in range(2))
    for s in range(w.shape[0]):
        a, b = offsets[s], offsets[s + 1]
        y[a:b] = x[a:b] @ w[s].T
        mag[a:b] = np.abs(x[a:b]) @ np.abs(w[s]).T
    return y, mag


def product_backward(dy, x, w, offsets):
    """((dx, magnitude), (dw, magnitude))."""
    dx, mx = np.zeros(x.shape), np.zeros(x.shape)
    dw, mw = np.zeros(w.shape), np.zeros(w.shape)
    for s in range(w.shape[0]):
        a, b = offsets[s], offsets[s + 1]
        dx[a:b], mx[a:b] = dy[a:b] @ w[s], np.abs(dy[a:b]) @ np.abs(w[s])
        dw[s], mw[s] = dy[a:b].T @ x[a:b], np.abs(dy[a:b]).T @ np.abs(x[a:b])
    return (dx, mx), (dw, mw)


def combine(y, places, gates):
    """(out, magnitude)."""
    on = (places >= 0) & (places < y.shape[0])
    part = np.where(on[..., None], y[np.where(on, places, 0)] * gates[..., None], 0.0)
    return part.sum(axis=1), np.abs(part).sum(axis=1)


def combine_backward(dout, y, rows, places, gates):
    """(dy, (dgates, magnitude))."""
    T, k = places.shape
    dy = np.zeros(y.shape)
    for r, p in enumerate(rows):
        if 0 <= p < T * k and places[p // k, p % k] == r:
            dy[r] = gates[p // k, p % k] * dout[p // k]
    on = (places >= 0) & (places < y.shape[0])
    part = np.where(on[..., None], y[np.where(on, places, 0)] * dout[:, None, :], 0.0)
    return dy, (part.sum(axis=-1), np.abs(part).sum(axis=-1))
