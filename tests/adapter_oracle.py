"""Low-rank adapters in 64 bits on the host, written from the formulas in include/bitlogic.h,
and rows by group."""
import numpy as np


def forward(x, down, up, ids, scales, base, base_scale):
    """(out, hidden, sizes): sizes bound what roundings of out's terms are relative to."""
    n, c, r = x.shape[0], up.shape[1], down.shape[1]
    out = np.zeros((n, c)) if base is None else base * base_scale
    sizes = np.abs(out)
    hidden = np.zeros((n, r))
    for s in range(n):
        a = ids[s]
        if 0 <= a < len(down):
            hidden[s] = down[a] @ x[s]
            out[s] += scales[a] * (up[a] @ hidden[s])
            sizes[s] += np.abs(scales[a]) * (np.abs(up[a]) @ (np.abs(down[a]) @ np.abs(x[s])))
    return out, hidden, sizes


def backward(grad, x, down, up, ids, scales):
    """Gradients of x, down and up, each with its sizes."""
    gx, gd, gu = np.zeros(x.shape), np.zeros(down.shape), np.zeros(up.shape)
    sx, sd, su = np.zeros(x.shape), np.zeros(down.shape), np.zeros(up.shape)
    for s in range(len(x)):
        a = ids[s]
        if not 0 <= a < len(down):
            continue
        k, size = scales[a], abs(scales[a])
        back, h = up[a].T @ grad[s], down[a] @ x[s]
        back_size, h_size = np.abs(up[a]).T @ np.abs(grad[s]), np.abs(down[a]) @ np.abs(x[s])
        gx[s] = k * (down[a].T @ back)
        sx[s] = size * (np.abs(down[a]).T @ back_size)
        gd[a] += k * np.outer(back, x[s])
        sd[a] += size * np.outer(back_size, np.abs(x[s]))
        gu[a] += k * np.outer(grad[s], h)
        su[a] += size * np.outer(np.abs(grad[s]), h_size)
    return (gx, sx), (gd, sd), (gu, su)


def groups(ids, n_groups):
    """(rows in the order of their groups, starts): rows without a group at the end."""
    ids = np.where((ids >= 0) & (ids < n_groups), ids, n_groups)
    return np.argsort(ids, kind="stable"), np.concatenate(
        [[0], np.cumsum(np.bincount(ids, minlength=n_groups + 1))])
