"""Plain 64-bit statements of the operators on paged caches and of the log probabilities (numpy)."""
import numpy as np


def slots(table, page, n):
    """(page, slot in it) of a sequence's first n tokens."""
    j = np.arange(n)
    return np.asarray(table)[j // page], j % page


def rotate(x, gain, eps, c, s):
    """x [heads, dh] of one row -> (rotated, sum of the products' magnitudes); c, s [dh / 2]."""
    x = np.asarray(x, dtype=np.float64)
    if gain is not None:
        x = x / np.sqrt(np.mean(x * x, -1, keepdims=True) + eps) * gain
    a, b = np.split(x, 2, -1)
    return (np.concatenate([a * c - b * s, b * c + a * s], -1),
            np.concatenate([np.abs(a * c) + np.abs(b * s), np.abs(b * c) + np.abs(a * s)], -1))


def attention_row(q, k, v, there=None):
    """One row and head over keys k [n, dh]: (output, sum of w |v|); keys where `there` is False are not seen."""
    if there is not None:
        k, v = k[there], v[there]
    if len(k) == 0:
        return np.zeros_like(q), np.zeros_like(q)
    x = (k @ q) * len(q) ** -0.5
    w = np.exp(x - x.max())
    w /= w.sum()
    return w @ v, w @ np.abs(v)


def logprobs(x, token, n_top):
    """One row: (log p of the token, entropy, rank, ids, their log p)."""
    x = np.asarray(x, dtype=np.float64)
    with np.errstate(invalid="ignore", divide="ignore"):
        m = np.nanmax(x) if not np.all(np.isnan(x)) else np.nan
        lp = (x - m) - np.log(np.sum(np.exp(x - m)))   # m first: beside the largest numbers a type holds, log V would be lost
        p = np.exp(lp)
        entropy = -np.sum(np.where(p == 0, 0.0, p * lp))
    order = sorted(range(len(x)), key=lambda j: (np.isnan(x[j]), -x[j] if not np.isnan(x[j]) else 0.0, j))
    top = order[:n_top]
    if token < 0:
        return 0.0, entropy, -1, top, lp[top]
    rank = -1 if np.isnan(x[token]) else int(np.sum(x > x[token]) + np.sum(x[:token] == x[token]))
    return lp[token], entropy, rank, top, lp[top]
