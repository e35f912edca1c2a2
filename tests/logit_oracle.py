"""Rows of class scores or logits in 64 bits on the host, written from the
definitions in include/bitlogic.h: the order of a row, top logits, the distillation
loss with its gradient, and sampling.  Inputs are numpy arrays of float64 (every
16- and 32-bit value is exact there); `masked` marks classes outside the order."""
import numpy as np


def order(x, masked):
    """Classes of one row by descending logit, then ascending class; no masked ones."""
    cls = np.nonzero(~masked)[0]
    return cls[np.argsort(-x[cls], kind="stable")]


def log_sum(x):
    """log sum e^x along the last axis; -inf where nothing is above -inf."""
    m = np.max(x, axis=-1, keepdims=True)
    m0 = np.where(np.isfinite(m), m, 0.0)
    with np.errstate(divide="ignore", over="ignore"):
        s = np.log(np.sum(np.exp(x - m0), axis=-1)) + m0[..., 0]
    return np.where(m[..., 0] == np.inf, np.inf, s)


def top(x, masked, k, temperature):
    """(classes [n][k], -1 past the last; log-normalizers [n])."""
    cls = np.full((x.shape[0], k), -1)
    for r in range(x.shape[0]):
        o = order(x[r], masked[r])[:k]
        cls[r, :len(o)] = o
    return cls, log_sum(np.where(masked, -np.inf, x) / temperature)


def distill(z, temperature, t, idx, top_temperature, log_norm=None):
    """One row: (loss, gradient, p, q over all classes, q_rest, p_rest)."""
    n = z.shape[0]
    have = (idx >= 0) & (idx < n)
    at, y = idx[have], t[have] / top_temperature
    with np.errstate(all="ignore"):
        log_p = z / temperature - log_sum(z / temperature)
        p = np.exp(log_p)
        norm = (log_sum(y) if len(y) else 0.0) if log_norm is None else log_norm
        qj = np.exp(y - norm)
        q = np.zeros(n)
        q[at] = qj
        use = qj != 0
        loss = np.sum(qj[use] * ((y - norm)[use] - log_p[at][use]))
        out = np.ones(n, bool)
        out[at] = False
        q_rest = 0.0 if log_norm is None else max(0.0, 1 - qj.sum())
        log_rest = log_sum(log_p[out]) if out.any() else -np.inf   # (p itself may vanish)
        p_rest = np.exp(log_rest)
        grad = (qj.sum() + q_rest) * p - q
        if q_rest > 0:
            loss += q_rest * (np.log(q_rest) - log_rest)
            if log_rest > -np.inf or np.isnan(log_rest) or not np.isfinite(z).any():
                grad[out] -= q_rest * np.exp(log_p[out] - log_rest)
        if qj.sum() + q_rest == 0:
            grad[:] = 0.0
    return loss, grad / temperature, p, q, q_rest, p_rest


def sample(x, masked, g, temperature, k, top_p, min_p, slack=0.0):
    """One row: (token, log_prob, kept classes).  Differences and products of x are
    rounded to 32 bits as defined; sums are not.  slack moves the top-p target and the
    min-p bound by that share: where rounding may decide, several answers are right."""
    o = order(x, masked)
    if len(o) == 0:
        return -1, -np.inf, o
    if not temperature > 0:
        return o[0], 0.0, o[:1]
    inv = np.float32(1) / np.float32(temperature)
    with np.errstate(invalid="ignore", over="ignore"):
        d = np.float32(x[o]) - np.float32(x[o[0]])
        y = np.where(x[o] == x[o[0]], np.float32(0), d * inv).astype(np.float64)
    if k > 0:
        o, y = o[:k], y[:k]
    w = np.exp(y)
    if top_p < 1:
        before = np.concatenate([[0.0], np.cumsum(w)[:-1]])
        keep = before < top_p * w.sum() * (1 + slack)
        keep[0] = True
        o, y, w = o[keep], y[keep], w[keep]
    if min_p > 0:
        keep = y >= np.log(min_p) * (1 + slack)
        keep[0] = True
        o, y, w = o[keep], y[keep], w[keep]
    score = (np.float32(y) + np.float32(g[o])).astype(np.float64)
    score = np.where(np.isnan(score), -np.inf, score)
    best = score.max()
    at = 0 if best == -np.inf else np.nonzero(score == best)[0][np.argmin(o[score == best])]
    return o[at], y[at] - np.log(w.sum()), o
