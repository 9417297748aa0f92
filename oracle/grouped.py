"""Plain float64 forms of the operators on weights in stacks: rows sorted by group, grouped products and their gradients."""
import numpy as np


def group_rows(group, n_groups):
    """(offsets [n_groups + 1], rows in the order of their groups)"""
    lists = [[] for _ in range(n_groups)]
    for r, g in enumerate(group):
        if 0 <= g < n_groups:
            lists[int(g)].append(r)
    ptr = [0]
    for rows in lists:
        ptr.append(ptr[-1] + len(rows))
    return np.array(ptr), np.array([r for rows in lists for r in rows], dtype=np.int64)


def linear(x, ptr, rows, w, bias=None):
    """{row: (y, sum of the terms' sizes)} as two arrays [rows, n_out] and which rows belong to a group"""
    y, size = (np.zeros((len(x), w.shape[2])) for _ in range(2))
    used = np.zeros(len(x), bool)
    for g in range(len(w)):
        r = rows[ptr[g]:ptr[g + 1]]
        with np.errstate(all="ignore"):
            y[r] = x[r] @ w[g] + (0.0 if bias is None else bias[g])
            size[r] = np.abs(x[r]) @ np.abs(w[g]) + (0.0 if bias is None else np.abs(bias[g]))
        used[r] = True
    return y, size, used


def linear_grad(x, ptr, rows, w, dy):
    """dx, dw, db, each with the sum of the sizes of its terms"""
    dx, dxs = (np.zeros(x.shape) for _ in range(2))
    dw, dws = (np.zeros(w.shape) for _ in range(2))
    db, dbs = (np.zeros((len(w), w.shape[2])) for _ in range(2))
    with np.errstate(all="ignore"):
        for g in range(len(w)):
            r = rows[ptr[g]:ptr[g + 1]]
            a, d = x[r], dy[r]
            dx[r], dxs[r] = d @ w[g].T, np.abs(d) @ np.abs(w[g]).T
            dw[g], dws[g] = a.T @ d, np.abs(a).T @ np.abs(d)
            db[g], dbs[g] = d.sum(0), np.abs(d).sum(0)
    return (dx, dxs), (dw, dws), (db, dbs)
