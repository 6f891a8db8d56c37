"""The balance loss and the router's gradient from their definitions, in 64 bits, and how far fp32 may be off."""
import numpy as np

EPS = 2.0 ** -24


def softmax(l):
    m = l.max(axis=1, keepdims=True)
    with np.errstate(invalid="ignore"):
        p = np.exp(l - np.where(np.isfinite(m), m, 0.0))
    s = p.sum(axis=1, keepdims=True)
    return p / np.where(s > 0, s, 1.0)


def groups_of(T, group):
    return [np.arange(T)] if group == 0 else [np.arange(a, min(T, a + group)) for a in range(0, T, group)]


def balance(logits, idx, mask, group, E, k):
    """(loss [G], counts [G, E], probs [G, E], n_tokens [G])."""
    out = ([], [], [], [])
    for rows in groups_of(len(logits), group):
        rows = rows if mask is None else rows[mask[rows] != 0]
        n = len(rows)
        picks = idx[rows].reshape(-1)
        c = np.bincount(picks[(picks >= 0) & (picks < E)], minlength=E)
        p = softmax(logits[rows].astype(np.float64)).sum(axis=0) / max(n, 1) if n else np.zeros(E)
        for o, v in zip(out, (E / (k * max(n, 1)) * (c @ p), c, p, n)):
            o.append(v)
    return tuple(np.array(o) for o in out)


def backward(logits, idx, mask, group, E, k, d_loss, d_gate, mode):
    """(d_logits [T, E], the magnitude of the terms that each element is the sum of)."""
    T = len(logits)
    d, size = np.zeros((T, E)), np.zeros((T, E))
    for g, rows in enumerate(groups_of(T, group)):
        rows = rows if mask is None else rows[mask[rows] != 0]
        n = len(rows)
        if n == 0:
            continue
        l = logits[rows].astype(np.float64)
        p = softmax(l)
        u = np.zeros((n, E))
        if d_loss is not None:
            picks = idx[rows].reshape(-1)
            c = np.bincount(picks[(picks >= 0) & (picks < E)], minlength=E).astype(np.float64)
            u += float(d_loss[g]) * E / (k * n * n) * (c - c.mean())
        # a rounded sum is off by EPS of the magnitudes of its terms at each addition, not of the sum: an expert picked more than once
        # adds several gate gradients to u, which may cancel
        u_size = np.abs(u)
        direct, direct_size = np.zeros((n, E)), np.zeros((n, E))
        if d_gate is not None:
            for t, row in enumerate(rows):
                js = [j for j in range(k) if 0 <= idx[row, j] < E]
                dg = d_gate[row, js].astype(np.float64)
                es = idx[row, js]
                if mode == "softmax_all":
                    np.add.at(u[t], es, dg)
                    np.add.at(u_size[t], es, np.abs(dg))
                elif js:
                    gate = softmax(l[t, es][None])[0]
                    np.add.at(direct[t], es, gate * (dg - gate @ dg))
                    np.add.at(direct_size[t], es, gate * (np.abs(dg) + gate @ np.abs(dg)))
        d[rows] = p * (u - (u * p).sum(axis=1, keepdims=True)) + direct
        size[rows] = p * (u_size + (u_size * p).sum(axis=1, keepdims=True)) + direct_size
    return d, size


def relative_error_of_p(spread):
    """Of a softmax in fp32 whose logits span `spread`: a difference to the maximum is rounded (half an ulp of at most
    `spread`) and so is its product with log2 e inside the exponential (the same again), the exponential is within 2 ulp, the
    sum of them has the same error and up to 8 additions and lane exchanges, a division and a product."""
    return (2 * (2 * spread + 2) + 8 + 2) * EPS
