"""CPU oracle of the calls on batches whose rows go to different weights: plain double-precision numpy, row by row, sharing no code with the
CUDA path.  TEST INFRASTRUCTURE ONLY.

* ``group_rows``      the plan of a batch.
* ``grouped``         experts' products, from dequantised matrices, with the sum of the products' magnitudes for error bounds.
* ``adapters``        what low-rank adapters add, and what error bounds need: t, and the magnitudes of its and the result's terms.
* ``adapters_grad``   their backward pass, the same.
"""
from __future__ import annotations

import numpy as np


def group_rows(group, G):
    group = [int(g) for g in np.asarray(group).reshape(-1)]
    order, groups, offsets = [], [], [0]
    for g in range(G):
        mine = [i for i, v in enumerate(group) if v == g]
        order += mine
        groups += [g] * len(mine)
        offsets.append(len(order))
    rest = [i for i, v in enumerate(group) if not 0 <= v < G]
    return np.array(order + rest, dtype=np.int64), np.array(groups + [-1] * len(rest), dtype=np.int64), np.array(offsets, dtype=np.int64)


def grouped(x, w, group, k):
    """x [T, K] and w [G, N, K] as what their codes stand for, group [T * k] -> (y [T * k, N], magnitudes [T * k, N])."""
    y, size = np.zeros((len(group), w.shape[1])), np.zeros((len(group), w.shape[1]))
    for p, g in enumerate(group):
        if 0 <= g < w.shape[0]:
            y[p] = w[g] @ x[p // k]
            size[p] = np.abs(w[g]) @ np.abs(x[p // k])
    return y, size


def adapters(x, a, b, group, base=None, scale=None):
    """-> (y, t, magnitudes of t's terms, of y's terms with t, of y's terms with t's magnitudes)."""
    M, G, r, N = x.shape[0], a.shape[0], a.shape[1], b.shape[1]
    y = np.zeros((M, N)) if base is None else base.copy()
    t, t_size, y_size, y_deep = np.zeros((M, r)), np.zeros((M, r)), np.zeros((M, N)), np.zeros((M, N))
    for m in range(M):
        g = int(group[m])
        if not 0 <= g < G:
            continue
        s = 1.0 if scale is None else float(scale[g])
        t[m] = a[g] @ x[m]
        t_size[m] = np.abs(a[g]) @ np.abs(x[m])
        y[m] += s * (b[g] @ t[m])
        y_size[m] = abs(s) * (np.abs(b[g]) @ np.abs(t[m]))
        y_deep[m] = abs(s) * (np.abs(b[g]) @ t_size[m])
    return y, t, t_size, y_size, y_deep


def adapters_grad(dy, x, a, b, t, group, base=None, scale=None):
    """-> ((dx, terms with dt, terms with dt's magnitudes), (da, the same), (db, terms))."""
    M, G, r, K, N = x.shape[0], a.shape[0], a.shape[1], a.shape[2], b.shape[1]
    dx = np.zeros((M, K)) if base is None else base.copy()
    dx_size, dx_deep = np.zeros((M, K)), np.zeros((M, K))
    da, da_size, da_deep = np.zeros((G, r, K)), np.zeros((G, r, K)), np.zeros((G, r, K))
    db, db_size = np.zeros((G, N, r)), np.zeros((G, N, r))
    for m in range(M):
        g = int(group[m])
        if not 0 <= g < G:
            continue
        s = 1.0 if scale is None else float(scale[g])
        dt, deep = s * (dy[m] @ b[g]), abs(s) * (np.abs(dy[m]) @ np.abs(b[g]))
        dx[m] += dt @ a[g]
        dx_size[m] = np.abs(dt) @ np.abs(a[g])
        dx_deep[m] = deep @ np.abs(a[g])
        da[g] += np.outer(dt, x[m])
        da_size[g] += np.outer(np.abs(dt), np.abs(x[m]))
        da_deep[g] += np.outer(deep, np.abs(x[m]))
        db[g] += s * np.outer(dy[m], t[m])
        db_size[g] += abs(s) * np.outer(np.abs(dy[m]), np.abs(t[m]))
    return (dx, dx_size, dx_deep), (da, da_size, da_deep), (db, db_size)
