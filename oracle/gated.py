"""fp64 statement of the gated linear recurrence, step by step.

Time first: x, r, i, z, y [T, B, D]; decay, r_bias, i_bias [D]; h0 [B, D]; lengths [B].
"""
import numpy as np

from .ssm import _lengths, sigmoid


def scan(x, r, i, decay, z=None, r_bias=None, i_bias=None, h0=None, lengths=None):
    """(y, last states, all states [T + 1, B, D])."""
    T, B, D = x.shape
    n = _lengths(lengths, T, B)
    h = np.zeros((T + 1, B, D))
    if h0 is not None:
        h[0] = h0
    y = np.zeros((T, B, D))
    for t in range(T):
        h[t + 1] = h[t]
        on = t < n
        size = decay * sigmoid(r[t, on] + (0.0 if r_bias is None else r_bias))
        iota = sigmoid(i[t, on] + (0.0 if i_bias is None else i_bias))
        h[t + 1, on] = np.exp(-size) * h[t, on] + np.sqrt(-np.expm1(-2 * size)) * iota * x[t, on]
        y[t, on] = h[t + 1, on] if z is None else h[t + 1, on] * z[t, on] * sigmoid(z[t, on])
    return y, h[T], h


def scan_backward(dy, x, r, i, decay, z=None, r_bias=None, i_bias=None, h0=None, lengths=None, dh_last=None):
    """Gradients of sum(y dy) + sum(h_last dh_last) as a dict."""
    T, B, D = x.shape
    _, _, h = scan(x, r, i, decay, z, r_bias, i_bias, h0, lengths)
    n = _lengths(lengths, T, B)
    g = {k: np.zeros((T, B, D)) for k in ("dx", "dr", "di", "dz")}
    g.update({k: np.zeros(D) for k in ("ddecay", "dr_bias", "di_bias")})
    carry = np.zeros((B, D)) if dh_last is None else np.array(dh_last, dtype=np.float64)
    for t in reversed(range(T)):
        on = np.flatnonzero(t < n)
        if not len(on):
            continue
        rho = sigmoid(r[t, on] + (0.0 if r_bias is None else r_bias))
        iota = sigmoid(i[t, on] + (0.0 if i_bias is None else i_bias))
        size = decay * rho
        a, m = np.exp(-size), np.sqrt(-np.expm1(-2 * size))
        q = dy[t, on]
        if z is not None:
            zt = z[t, on]
            sg = sigmoid(zt)
            g["dz"][t, on] = q * h[t + 1, on] * sg * (1 + zt * (1 - sg))
            q = q * zt * sg
        G = q + carry[on]
        with np.errstate(divide="ignore"):
            over = np.where(m > 0, 1 / m, 0.0)
        # through the decay: da = -a dsize, dm = a^2 / m dsize
        dsize = G * (a * a * over * iota * x[t, on] - a * h[t, on])
        carry[on] = a * G
        g["dx"][t, on] = G * m * iota
        g["di"][t, on] = G * m * x[t, on] * iota * (1 - iota)
        g["dr"][t, on] = dsize * decay * rho * (1 - rho)
        g["ddecay"] += (dsize * rho).sum(0)
        g["dr_bias"] += g["dr"][t, on].sum(0)
        g["di_bias"] += g["di"][t, on].sum(0)
    g["dh0"] = carry
    return g
