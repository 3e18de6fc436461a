"""fp64 statement of the loss against a teacher's top logits, row by row.

logits [R, V]; top_logits, top_index [R, K]; top_norm, weight, targets [R].
"""
import numpy as np


def _log_softmax(x):
    m = np.max(x)
    with np.errstate(invalid="ignore"):        # a largest value that is infinite: NaN
        return x - (m + np.log(np.sum(np.exp(x - m))))


def loss(logits, top_logits, top_index, temperature=1.0, top_norm=None, targets=None, hard=0.0, weight=None):
    """(loss [R], dlogits [R, V])."""
    R, V = logits.shape
    out, grad = np.zeros(R), np.zeros((R, V))
    for k in range(R):
        w = 1.0 if weight is None else weight[k]
        if w == 0:
            continue
        on = (top_index[k] >= 0) & (top_index[k] < V) & (top_logits[k] != -np.inf)       # NaN counts
        c, t = top_index[k][on], top_logits[k][on] / temperature
        logq = _log_softmax(logits[k] / temperature)
        q = np.exp(logq)
        soft, d = 0.0, np.zeros(V)
        if len(c):
            logp = _log_softmax(t) if top_norm is None else t - top_norm[k]
            p = np.exp(logp)
            soft = np.sum(np.where(p == 0, 0.0, p * (logp - logq[c])))
            d = q * p.sum()
            with np.errstate(invalid="ignore"):
                np.subtract.at(d, c, p)
        if top_norm is not None:
            rest = np.ones(V, dtype=bool)
            rest[c] = False
            p0, q0 = np.maximum(0.0, 1.0 - (p.sum() if len(c) else 0.0)), q[rest].sum()
            if p0 != 0 and q0 > 0:
                soft += p0 * np.log(p0 / q0)
                d += p0 * q
                d[rest] -= p0 * q[rest] / q0
        out[k] = (1 - hard) * temperature ** 2 * soft
        grad[k] = (1 - hard) * temperature * d
        if hard and 0 <= targets[k] < V:
            logq = _log_softmax(logits[k])
            out[k] -= hard * logq[targets[k]]
            grad[k] += hard * np.exp(logq)
            grad[k, targets[k]] -= hard
        out[k] *= w
        grad[k] *= w
    return out, grad
