"""fp64 statement of the selective state space layer and of the AdamW update over tensors, step by step.

Time first: u, dt, z, y [T, B, D]; Bm, Cm [T, B, G, N]; A [D, N]; skip, dt_bias [D]; h0 [B, D, N]; lengths [B].
"""
import numpy as np


def softplus(x):
    return np.logaddexp(0.0, x)


def sigmoid(x):
    return np.exp(-np.logaddexp(0.0, -x))


def _lengths(lengths, T, B):
    return np.full(B, T) if lengths is None else np.clip(np.asarray(lengths, dtype=np.int64), 0, T)


def scan(u, dt, A, Bm, Cm, skip=None, z=None, dt_bias=None, h0=None, lengths=None):
    """(y, last states, all states [T + 1, B, D, N], the output before the gate)."""
    T, B, D = u.shape
    G, N = Bm.shape[2:]
    of = np.arange(D) // (D // G)
    skip = np.zeros(D) if skip is None else skip
    bias = np.zeros(D) if dt_bias is None else dt_bias
    n = _lengths(lengths, T, B)
    h = np.zeros((T + 1, B, D, N))
    if h0 is not None:
        h[0] = h0
    y, plain = np.zeros((T, B, D)), np.zeros((T, B, D))
    for t in range(T):
        h[t + 1] = h[t]
        on = t < n
        s = softplus(dt[t, on] + bias)[..., None]
        h[t + 1, on] = np.exp(s * A) * h[t, on] + s * u[t, on][..., None] * Bm[t, on][:, of]
        plain[t, on] = (h[t + 1, on] * Cm[t, on][:, of]).sum(-1) + skip * u[t, on]
        y[t, on] = plain[t, on] if z is None else plain[t, on] * z[t, on] * sigmoid(z[t, on])
    return y, h[T], h, plain


def scan_backward(dy, u, dt, A, Bm, Cm, skip=None, z=None, dt_bias=None, h0=None, lengths=None):
    """Gradients of sum(y dy) as a dict."""
    T, B, D = u.shape
    G, N = Bm.shape[2:]
    of = np.arange(D) // (D // G)
    _, _, h, plain = scan(u, dt, A, Bm, Cm, skip, z, dt_bias, h0, lengths)
    skip = np.zeros(D) if skip is None else skip
    bias = np.zeros(D) if dt_bias is None else dt_bias
    n = _lengths(lengths, T, B)
    g = {"du": np.zeros((T, B, D)), "ddt": np.zeros((T, B, D)), "dz": np.zeros((T, B, D)), "dBm": np.zeros((T, B, G, N)),
         "dCm": np.zeros((T, B, G, N)), "dA": np.zeros((D, N)), "dskip": np.zeros(D), "ddt_bias": np.zeros(D)}
    carry = np.zeros((B, D, N))
    for t in reversed(range(T)):
        on = np.flatnonzero(t < n)
        if not len(on):
            continue
        raw = dt[t, on] + bias
        s, x, q = softplus(raw), u[t, on], dy[t, on]
        if z is not None:
            zt = z[t, on]
            sg = sigmoid(zt)
            g["dz"][t, on] = q * plain[t, on] * sg * (1 + zt * (1 - sg))
            q = q * zt * sg
        G_h = q[..., None] * Cm[t, on][:, of] + carry[on]
        g["dCm"][t, on] = (h[t + 1, on] * q[..., None]).reshape(len(on), G, D // G, N).sum(2)
        g["dBm"][t, on] = (G_h * (s * x)[..., None]).reshape(len(on), G, D // G, N).sum(2)
        carry[on] = np.exp(s[..., None] * A) * G_h
        through = carry[on] * h[t, on]
        s1 = (G_h * Bm[t, on][:, of]).sum(-1)
        g["du"][t, on] = s * s1 + skip * q
        ddt = (x * s1 + (through * A).sum(-1)) * sigmoid(raw)
        g["ddt"][t, on] = ddt
        g["ddt_bias"] += ddt.sum(0)
        g["dA"] += (through * s[..., None]).sum(0)
        g["dskip"] += (q * x).sum(0)
    g["dh0"] = carry
    return g


def conv(x, weight, bias=None, silu=True, state0=None, lengths=None):
    """(y, last W - 1 inputs of each sample, p before the silu, the row of inputs with the state in front [T + W - 1, B, D])."""
    T, B, D = x.shape
    W = weight.shape[1]
    n = _lengths(lengths, T, B)
    inside = (np.arange(T)[:, None] < n)[..., None]
    row = np.zeros((T + W - 1, B, D))
    if state0 is not None:
        row[:W - 1] = np.moveaxis(state0, 1, 0)
    row[W - 1:] = np.where(inside, x, 0.0)
    p = sum(weight[:, k] * row[k:k + T] for k in range(W)) + (0.0 if bias is None else bias)
    y = np.where(inside, p * sigmoid(p) if silu else p, 0.0)
    last = np.stack([row[k:k + W - 1, b] for b, k in enumerate(n)])
    return y, last, p, row


def conv_backward(dy, x, weight, bias=None, silu=True, state0=None, lengths=None):
    T, B, D = x.shape
    W = weight.shape[1]
    _, _, p, row = conv(x, weight, bias, silu, state0, lengths)
    inside = (np.arange(T)[:, None] < _lengths(lengths, T, B))[..., None]
    dp = np.where(inside, dy, 0.0)
    if silu:
        sg = sigmoid(p)
        dp = dp * sg * (1 + p * (1 - sg))
    drow = np.zeros_like(row)
    for k in range(W):
        drow[k:k + T] += weight[:, k] * dp
    return {"dx": np.where(inside, drow[W - 1:], 0.0), "dstate0": np.moveaxis(drow[:W - 1], 0, 1),
            "dweight": np.stack([(dp * row[k:k + T]).sum((0, 1)) for k in range(W)], 1), "dbias": dp.sum((0, 1))}


def adamw(theta, grad, m, v, step, lr, beta1, beta2, eps, decay):
    """(theta, m, v) after one update."""
    m = beta1 * m + (1 - beta1) * grad
    v = beta2 * v + (1 - beta2) * grad ** 2
    return (theta * (1 - lr * decay) - lr * (m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps)), m, v


def e4m3_values():
    """The 127 magnitudes of e4m3, ascending: seven subnormals above zero, then eight to each power of two, 448 the last."""
    sub = np.arange(8) * 2.0 ** -9
    rest = [(1 + k / 8) * 2.0 ** e for e in range(-6, 9) for k in range(8)]
    return np.concatenate([sub, rest])[:127]


def _numbers(seed, tensor, n):
    low = 0xFFFFFFFF
    x = (np.arange(n, dtype=np.uint64) + np.uint64((seed * 0x9E3779B1 + tensor * 0x6A09E667) & low)) & np.uint64(low)
    for k in (0xBB67AE85, 0x3C6EF373):
        x = ((x ^ (x >> np.uint64(16))) * np.uint64(k)) & np.uint64(low)
    return x ^ (x >> np.uint64(15))


def chance(seed, tensor, n):
    """[0, 1) for places 0..n of a tensor: two rounds of multiply and fold over place, tensor and seed."""
    return (_numbers(seed, tensor, n) >> np.uint64(8)).astype(np.float64) * 2.0 ** -24


def chance_of_m(seed, tensor, n):
    """The same for the first moment, where that is rounded by chance."""
    x = (_numbers(seed, tensor, n) * np.uint64(0x9E3779B1)) & np.uint64(0xFFFFFFFF)
    return (x >> np.uint64(8)).astype(np.float64) * 2.0 ** -24


def held_m(q, shrinks, beta1, by):
    """e4m3 values of first moments q in units of their scales; `shrinks`: the magnitude has become smaller, `by`: [0, 1) each.
    Also which of them went by chance."""
    grid, size = e4m3_values(), np.clip(np.abs(q), 0, 448)
    above = np.clip(np.searchsorted(grid, size), 1, 126)
    lo, hi = grid[above - 1], grid[above]
    share = (size - lo) / (hi - lo)
    by_chance = (shrinks & (size < 2.0 ** -6)) | (beta1 > 15 / 16)
    nearest = np.where((share < 0.5) | ((share == 0.5) & (above % 2 == 1)), lo, hi)
    return np.sign(q) * np.where(by_chance, np.where(share + by >= 1, hi, lo), nearest), by_chance
