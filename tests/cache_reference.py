"""Plain 64-bit statements of the operators on bounded and shared caches, one row at a time (numpy)."""
import numpy as np


def softmax_row(q, K, scale):
    """Weights of one query over keys K [n, dh] (NaN / inf as the formula has them)."""
    x = (K @ q) * scale
    e = np.exp(x - np.max(x))
    return e / np.sum(e)


def attention_mass(q, k, lens, H, Hkv, dh, window):
    """q [n, H, dh], k [n, Hkv, dh] -> mass [Hkv, n]."""
    out = np.zeros((Hkv, q.shape[0]))
    a = 0
    for n in lens:
        for i in range(max(n - window, 0) if window else 0, n):
            for h in range(H):
                g = h // (H // Hkv)
                out[g, a:a + i + 1] += softmax_row(q[a + i, h], k[a:a + i + 1, g], dh ** -0.5)
        a += n
    return out


def weight_order(w):
    """Sort key of a weight: NaN below everything, -0 equal to 0."""
    return (0, 0.0) if np.isnan(w) else (1, float(w) + 0.0)


def kept_rows(mass, n, budget, recent):
    """Row indices (ascending) that one head of a sequence of n rows keeps."""
    keep = min(n, budget)
    old = n - min(recent, keep)
    # stable sort: among equal weights the lower row comes first
    ranked = sorted(range(old), key=lambda i: weight_order(mass[i]), reverse=False)
    best = sorted(ranked, key=lambda i: weight_order(mass[i]), reverse=True)
    return sorted(best[:keep - (n - old)]) + list(range(old, n))


def step_slot(mass, pos, length, budget, pos_new, recent):
    """(slot, evicted position or -1, length after the step) of one head."""
    if length < budget:
        return length, -1, length + 1
    free = [j for j in range(length) if pos[j] < pos_new - recent]
    slot = min(free, key=lambda j: (weight_order(mass[j]), j)) if free else 0
    return slot, int(pos[slot]), length


def prefix_visible(rows, own):
    """Own keys that row i of `rows` sees."""
    return [max(own - rows + i + 1, 0) for i in range(rows)]


def verify(p, q, draft, u_accept, u_sample):
    """One sequence: p [T + 1, V], q [T, V] or None -> (accepted, next token)."""
    T = len(draft)
    acc = 0
    while acc < T:
        x = int(draft[acc])
        qx = 1.0 if q is None else float(q[acc, x])
        if not float(u_accept[acc]) * qx < float(p[acc, x]):
            break
        acc += 1
    w = np.maximum(np.nan_to_num(p[acc].astype(np.float64), nan=0.0), 0.0)
    if acc < T:
        if q is None:
            r = w.copy()
            r[int(draft[acc])] = 0.0
        else:
            r = np.maximum(p[acc].astype(np.float64) - q[acc].astype(np.float64), 0.0)
        if r.sum() > 0:
            w = r
    if not w.sum() > 0:
        return acc, -1
    run = np.cumsum(w)
    above = np.nonzero(run > float(u_sample) * run[-1])[0]
    return acc, int(above[0])
