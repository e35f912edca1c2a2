"""Draft verification and dropout in 64 bits on the host, written from the definitions in
include/bitlogic.h.  Logits are numpy arrays of float64 (every 16- and 32-bit value is exact
there); masked classes are marked apart."""
import numpy as np


def shares(x, masked, temperature):
    """(log p of every class, largest logit's first class or -1) of one row; temperature 0:
    one at that class."""
    at = np.nonzero(~masked)[0]
    out = np.full(len(x), -np.inf)
    if not len(at):
        return out, -1
    m = x[at].max()
    first = at[np.argmax(x[at] == m)]
    if not temperature > 0:
        out[first] = 0.0
        return out, first
    with np.errstate(invalid="ignore", over="ignore"):
        y = np.where(x[at] == m, 0.0, (x[at] - m) / max(temperature, 2.0 ** -126))
    out[at] = y - np.log(np.exp(y).sum())
    return out, first


def verify(x, masked, drafted, y, y_masked, uniform, noise, temperature, draft_temperature):
    """One request: (accepted, token, log_prob).  x [len + 1][c], drafted [len], y [len][c] or
    None, uniform [len], noise [c]."""
    c, length = x.shape[1], len(drafted)
    for i in range(length + 1):
        log_p, first = shares(x[i], masked[i], temperature)
        mass = np.exp(log_p)
        if i < length:
            t = int(drafted[i])
            log_q = np.full(c, -np.inf)
            if y is not None and draft_temperature > 0:
                log_q, _ = shares(y[i], y_masked[i], draft_temperature)
            elif 0 <= t < c:
                log_q[t] = 0.0
            if 0 <= t < c and log_p[t] > -np.inf:
                with np.errstate(over="ignore"):
                    ratio = np.exp(log_p[t] - log_q[t])
                if (t == first) if not temperature > 0 else uniform[i] < ratio:
                    continue
            less = mass - np.exp(log_q)
            if (less > 0).any():
                mass = np.where(less > 0, less, 0.0)
        if first < 0:
            return i, -1, -np.inf
        if not temperature > 0:
            return i, first, 0.0
        with np.errstate(divide="ignore", invalid="ignore"):
            score = np.log(mass) + noise
        score = np.where(np.isnan(score) | (mass == 0), -np.inf, score)
        token = int(score.argmax()) if score.max() > -np.inf else first
        return i, token, log_p[token]


def numbers(rows, cols, seed, offset):
    """The 16-bit numbers of a mask, from the generator's definition with Python integers."""
    low = 0xFFFFFFFF
    out = np.empty((rows, (cols + 7) // 8 * 8), np.int64)
    for s in range(rows):
        for block in range((cols + 7) // 8):
            c = [block, s, offset & low, offset >> 32 & low]
            k = [seed & low, seed >> 32]
            for _ in range(10):
                a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
                c = [b >> 32 ^ c[1] ^ k[0], b & low, a >> 32 ^ c[3] ^ k[1], a & low]
                k = [k[0] + 0x9E3779B9 & low, k[1] + 0xBB67AE85 & low]
            out[s, 8 * block:8 * block + 8] = [h for w in c for h in (w & 0xFFFF, w >> 16)]
    return out[:, :cols]


def dropout(x, p, seed, offset):
    """x float64 [rows][cols] -> what is kept, times its factor (in 64 bits)."""
    border = int(np.floor(float(np.float32(p)) * 65536 + 0.5))
    if border == 65536:
        return np.zeros_like(x)
    keep = numbers(*x.shape, seed, offset) >= border
    return np.where(keep, x * (65536 / (65536 - border)), 0.0)
