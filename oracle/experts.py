"""Cluster experts in fp64 from their definitions: assignment of rows to clusters, products by group, weighted sum, 8-bit blocks,
and the gradients.  Plain loops over rows and groups; shares nothing with the library."""
from __future__ import annotations

import numpy as np


def route(scores, t, allowed=None, normalize=True):
    """(idx, weight, p): the t best clusters of every row, their weights, and the softmax that the weights are taken from."""
    s = np.asarray(scores, dtype=np.float64)
    n, k = s.shape
    ok = ~(np.isnan(s) | (s == -np.inf))
    if allowed is not None:
        ok &= np.broadcast_to(np.asarray(allowed, dtype=bool), (n, k))
    idx = np.full((n, t), -1, dtype=np.int32)
    weight = np.zeros((n, t))
    p = np.zeros((n, k))
    for i in range(n):
        may = np.flatnonzero(ok[i])
        if may.size == 0:
            continue
        best = sorted(may, key=lambda j: (-s[i, j], j))[:t]
        idx[i, :len(best)] = best
        over = np.array(best) if normalize else may
        with np.errstate(invalid="ignore"):
            e = np.exp(s[i, over] - s[i, best[0]])
            p[i, over] = e / e.sum()
        weight[i, :len(best)] = p[i, best]
    return idx, weight, p


def route_backward(idx, weight, p, dweight):
    n, t = idx.shape
    ds = np.zeros_like(p)
    for i in range(n):
        c = 0.0
        for s in range(t):
            if idx[i, s] >= 0:
                c += weight[i, s] * dweight[i, s]
                ds[i, idx[i, s]] += p[i, idx[i, s]] * dweight[i, s]
        ds[i] -= p[i] * c
    return ds


def grouping(idx, k):
    """offsets, order, place of the slots with a cluster, by cluster, in slot order within a cluster."""
    flat = np.asarray(idx).reshape(-1)
    slots = [f for g in range(k) for f in np.flatnonzero(flat == g)]
    offsets = np.concatenate([[0], np.cumsum([(flat == g).sum() for g in range(k)])])
    order = np.full(flat.size, -1, dtype=np.int32)
    place = np.full(flat.size, -1, dtype=np.int32)
    order[:len(slots)] = slots
    place[order[:len(slots)]] = np.arange(len(slots))
    return offsets.astype(np.int32), order, place.reshape(np.shape(idx))


def _sources(x, order, slots, rows):
    """The rows of x that the grouped rows take; zeros where there is none."""
    x = np.asarray(x, dtype=np.float64)
    out = np.zeros((rows, x.shape[1]))
    for p in range(rows):
        r = p if order is None else (order[p] // slots if order[p] >= 0 else -1)
        if 0 <= r < x.shape[0]:
            out[p] = x[r]
    return out


def grouped_product(x, w, offsets, order=None, slots=1, transpose=False):
    """(y, |x| |w|): the second is what rounding errors are measured by."""
    w = np.asarray(w, dtype=np.float64)
    rows = len(x) if order is None else len(order)
    xs = _sources(x, order, slots, rows)
    y = np.zeros((rows, w.shape[2] if transpose else w.shape[1]))
    size = np.zeros_like(y)
    for g in range(w.shape[0]):
        a, b = offsets[g], offsets[g + 1]
        m = w[g] if transpose else w[g].T
        y[a:b] = xs[a:b] @ m
        size[a:b] = np.abs(xs[a:b]) @ np.abs(m)
    return y, size


def grouped_gradient(dy, x, offsets, order=None, slots=1):
    dy = np.asarray(dy, dtype=np.float64)
    xs = _sources(x, order, slots, len(dy))
    groups = len(offsets) - 1
    dw = np.zeros((groups, dy.shape[1], xs.shape[1]))
    size = np.zeros_like(dw)
    for g in range(groups):
        a, b = offsets[g], offsets[g + 1]
        dw[g] = dy[a:b].T @ xs[a:b]
        size[g] = np.abs(dy[a:b]).T @ np.abs(xs[a:b])
    return dw, size


def combine(z, place, weight=None):
    z = np.asarray(z, dtype=np.float64)
    n, t = place.shape
    out = np.zeros((n, z.shape[1]))
    size = np.zeros_like(out)
    for i in range(n):
        for s in range(t):
            if place[i, s] >= 0:
                term = (1.0 if weight is None else float(weight[i, s])) * z[place[i, s]]
                out[i] += term
                size[i] += np.abs(term)
    return out, size


def combine_backward(dout, z, place, weight=None):
    dout, z = np.asarray(dout, dtype=np.float64), np.asarray(z, dtype=np.float64)
    n, t = place.shape
    dz = np.zeros_like(z)
    dw = np.zeros((n, t))
    size = np.zeros((n, t))
    for i in range(n):
        for s in range(t):
            p = place[i, s]
            if p >= 0:
                dz[p] = (1.0 if weight is None else float(weight[i, s])) * dout[i]
                dw[i, s] = dout[i] @ z[p]
                size[i, s] = np.abs(dout[i]) @ np.abs(z[p])
    return dz, dw, size


def e4m3_values():
    """The values of codes 0 ... 126 (4 bits of exponent with bias 7, 3 of fraction)."""
    return np.array([(c & 7) / 8 * 2.0 ** -6 if c < 8 else (1 + (c & 7) / 8) * 2.0 ** ((c >> 3) - 7) for c in range(127)])


def quantize_blocks(x):
    """(codes uint8 (rows, Kp), exponent + 127 (rows, Kp / 128), values fp64 (rows, Kp)), every value looked up in the table."""
    x = np.asarray(x, dtype=np.float64)
    rows, K = x.shape
    nb = -(-K // 128)
    v = np.zeros((rows, nb * 128))
    v[:, :K] = x
    v = v.reshape(rows, nb, 128)
    finite = np.isfinite(v)
    most = np.where(finite, np.abs(v), 0.0).max(2)
    e = np.zeros((rows, nb), dtype=np.int64)
    for i in range(rows):
        for b in range(nb):
            if most[i, b] > 0:
                x2 = int(np.floor(np.log2(most[i, b]))) - 12
                while most[i, b] > 448.0 * 2.0 ** x2:
                    x2 += 1
                e[i, b] = max(x2, -127)
    tab = e4m3_values()
    a = np.where(finite, np.abs(v), 0.0) * 2.0 ** -e[:, :, None].astype(np.float64)
    hi = np.clip(np.searchsorted(tab, a), 0, 126)             # first code that is not smaller
    lo = np.maximum(hi - 1, 0)
    up, down = tab[hi] - a, a - tab[lo]
    code = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))
    val = np.where(np.signbit(v), -1.0, 1.0) * tab[code] * 2.0 ** e[:, :, None].astype(np.float64)
    code = np.where(np.signbit(v), code + 128, code)
    code = np.where(finite, code, np.where(np.signbit(v) & ~np.isnan(v), 255, 127))
    val = np.where(finite, val, np.nan)
    return code.astype(np.uint8).reshape(rows, -1), (e + 127).astype(np.uint8), val.reshape(rows, -1)
