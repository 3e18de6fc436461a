"""The selective state space layer's operators and the optimiser over many tensors, as cases that can be timed and compared.

Kinds, each a dict of plain values:

  scan_prompt  the selective scan over whole sequences, with the state after them: what serving does with a prompt.
  scan_train   the same scan forward and all its gradients: what a training step does with the layer.
  scan_token   one token of every running stream, the states held in slots of a cache and advanced in place.
  conv_prompt, conv_train, conv_token
               the short causal convolution in front of the scan, in the same three uses.
  adamw        one AdamW step over all tensors of a stack of such layers, moments in 32 bits or in 8.

Activations are float32, bfloat16 or float16; parameters, states and their gradients are float32.  Time comes first,
[T, B, channels], as everywhere in this package; `order` says how the memory lies ("tb": as the shape says, "bt": sequence
by sequence, the tensors are transposed views).  z, B and C are column slices of wider projections, as a layer has them.
`ragged`: the samples have lengths of their own; what lies behind a sample's end is padding of any value.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BLOCK = 256                                    # values that share a scale in the 8-bit moments
MOST = 4 * 4096 * 4096 * 16                    # state values (T B D N) of the largest scan


def listed():
    return [
        # The smallest prompt of the package's configurations: nothing but latency.
        {"name": "scan_prompt_T16_B2_D40", "kind": "scan_prompt", "T": 16, "B": 2, "D": 40, "N": 8, "G": 1, "type": "f32",
         "z": False, "h0": False, "ragged": False, "order": "tb"},
        # A batch of ordinary prompts of different lengths, sequence by sequence in memory, into a gated layer.
        {"name": "scan_prompt_T1000_B16_D640_bf16", "kind": "scan_prompt", "T": 1000, "B": 16, "D": 640, "N": 16, "G": 1,
         "type": "bf16", "z": True, "h0": False, "ragged": True, "order": "bt"},
        # One very long prompt: all the parallelism there is lies along the sequence.
        {"name": "scan_prompt_T30000_B1_D2048_bf16", "kind": "scan_prompt", "T": 30000, "B": 1, "D": 2048, "N": 16, "G": 1,
         "type": "bf16", "z": True, "h0": True, "ragged": False, "order": "tb"},
        # Training in float32 with ragged lengths, a channel count that no tile divides and two groups of B and C.
        {"name": "scan_train_T1000_B16_D330_f32", "kind": "scan_train", "T": 1000, "B": 16, "D": 330, "N": 16, "G": 2,
         "type": "f32", "z": False, "h0": True, "ragged": True, "order": "tb"},
        # The training step of a large gated layer.
        {"name": "scan_train_T4096_B4_D4096_bf16", "kind": "scan_train", "T": 4096, "B": 4, "D": 4096, "N": 16, "G": 1,
         "type": "bf16", "z": True, "h0": False, "ragged": False, "order": "tb"},
        # One token of 64 running streams.
        {"name": "scan_token_B64_D4096_bf16", "kind": "scan_token", "B": 64, "D": 4096, "N": 16, "G": 1, "type": "bf16",
         "z": True, "slots": 80},
        # The convolution in front of the large layer.
        {"name": "conv_prompt_T4096_B4_D4096_bf16", "kind": "conv_prompt", "T": 4096, "B": 4, "D": 4096, "W": 4,
         "type": "bf16", "silu": True, "state0": False, "ragged": False, "order": "tb"},
        # Its training step at an ordinary size in float16, ragged, with a state carried in.
        {"name": "conv_train_T1000_B16_D641_f16", "kind": "conv_train", "T": 1000, "B": 16, "D": 641, "W": 4,
         "type": "f16", "silu": True, "state0": True, "ragged": True, "order": "bt"},
        # One token of 64 running streams.
        {"name": "conv_token_B64_D4096_bf16", "kind": "conv_token", "B": 64, "D": 4096, "W": 4, "type": "bf16",
         "silu": True, "slots": 80},
        # The optimiser of a small stack: 80 tensors, most of them a few kilobytes.
        {"name": "adamw_32_L8_width128", "kind": "adamw", "layers": 8, "width": 128, "N": 16, "bits": 32, "grad": "f32",
         "copy": False},
        # The optimiser of a large stack: moments in 32 bits, bfloat16 gradients and working copies of the weights.
        {"name": "adamw_32_L8_width2048", "kind": "adamw", "layers": 8, "width": 2048, "N": 16, "bits": 32, "grad": "bf16",
         "copy": True},
        # The same stack with the moments in 8 bits.
        {"name": "adamw_8_L8_width2048", "kind": "adamw", "layers": 8, "width": 2048, "N": 16, "bits": 8, "grad": "bf16",
         "copy": True},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("scan_prompt", "scan_prompt", "scan_train", "scan_train", "scan_token", "conv_prompt", "conv_train",
                       "conv_token", "adamw"))
    case = {"kind": kind}
    if kind == "adamw":
        width = _log_int(rng, 20, 2048)
        most = max(1, min(24, int(8 * (2048 / width) ** 2)))
        return dict(case, layers=rng.randint(1, most), width=width, N=rng.choice((8, 16, 16, 64)), bits=rng.choice((32, 8)),
                    grad=rng.choice(("f32", "bf16", "f16")), copy=rng.random() < 0.5)
    case["type"] = rng.choice(("f32", "bf16", "bf16", "f16"))
    if kind in ("scan_token", "conv_token"):
        case["B"], case["D"] = _log_int(rng, 1, 256), _log_int(rng, 64, 8192)
        case["slots"] = case["B"] + rng.randint(0, 32)
        if kind == "conv_token":
            return dict(case, W=rng.choice((2, 3, 4, 4)), silu=rng.random() < 0.8)
        case["N"], case["G"] = rng.choice((4, 8, 16, 16, 16, 24, 32, 64)), rng.choice((1, 1, 1, 2, 4))
        case["D"] -= case["D"] % case["G"]
        return dict(case, z=rng.random() < 0.6)
    case["D"] = _log_int(rng, 16, 8192)
    N = rng.choice((4, 8, 16, 16, 16, 16, 24, 32, 64)) if kind.startswith("scan") else 16
    room = MOST // (case["D"] * N)
    case["T"] = _log_int(rng, 1, min(room, 4096 if kind.endswith("train") else 30000))
    case["B"] = _log_int(rng, 1, max(1, min(64, room // case["T"])))
    case["ragged"] = case["B"] > 1 and rng.random() < 0.4
    case["order"] = rng.choice(("tb", "bt"))
    if kind.startswith("conv"):
        return dict(case, W=rng.choice((2, 3, 4, 4)), silu=rng.random() < 0.8, state0=rng.random() < 0.4)
    G = rng.choice((1, 1, 1, 2, 4))
    case["D"] -= case["D"] % G
    return dict(case, N=N, G=G, z=rng.random() < 0.6, h0=rng.random() < 0.4)


# ---- inputs --------------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def _uniform(g, lo, hi, *shape):
    return lo + (hi - lo) * torch.rand(shape, generator=g, device=DEV)


def _rows(g, case, width):
    """[T, B, width] normal values of the case's type, in its order."""
    T, B = case["T"], case["B"]
    if case["order"] == "bt":
        return torch.randn((B, T, width), generator=g, device=DEV, dtype=TYPES[case["type"]]).transpose(0, 1)
    return torch.randn((T, B, width), generator=g, device=DEV, dtype=TYPES[case["type"]])


def _lengths(g, case):
    """Half to all of T, and one sample that is empty and one of a single token."""
    T, B = case["T"], case["B"]
    n = torch.randint((T + 1) // 2, T + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
    n[-1] = 1
    if B > 2:
        n[1] = 0
    return n


def _layer(g, D, N):
    """A, the skip weight and the step's bias as such a layer starts from: A = -1..-N, steps of 0.001 to 0.1."""
    A = -torch.arange(1, N + 1, device=DEV, dtype=torch.float32).expand(D, N) * _uniform(g, 0.8, 1.25, D, N)
    step = torch.exp(_uniform(g, math.log(1e-3), math.log(0.1), D))
    return A.contiguous(), _normal(g, D), step + torch.log(-torch.expm1(-step))


def _tensors(case):
    """(length, decayed) of each tensor of the stack: the two projections, convolution, step and state parameters, norm."""
    d, N = case["width"], case["N"]
    D, R = 2 * d, -(-d // 16)
    one = [(2 * D * d, True), (D * 4, False), (D, False), ((R + 2 * N) * D, True), (D * R, True), (D, False), (D * N, False),
           (D, False), (d * D, True), (d, False)]
    return one * case["layers"]


def prepare(case, seed):
    g, kind = _gen(seed), case["kind"]
    s = {"case": case, "kind": kind}
    if kind == "adamw":
        at, where = 0, []
        for n, decayed in _tensors(case):
            where.append((at, n, 0.1 if decayed else 0.0))
            at += -(-n // BLOCK) * BLOCK       # every tensor starts at a block of its own in the flat arrays
        real = torch.zeros(at, dtype=torch.bool, device=DEV)
        for o, n, _ in where:
            real[o:o + n] = True
        s["theta"] = torch.randn(at, generator=g, device=DEV).mul_(0.02).mul_(real)
        # gradients of very different sizes from block to block and within one
        size = torch.exp(_uniform(g, -9.0, -3.0, at // BLOCK, 1)) * torch.exp(_normal(g, at // BLOCK, BLOCK))
        grad = (_normal(g, at // BLOCK, BLOCK) * size).reshape(-1).mul_(real)
        s["grad"] = grad.to(TYPES[case["grad"]])
        m = _normal(g, at).mul_(0.3).mul_(size.reshape(-1)).mul_(real)
        v = _uniform(g, 0.3, 2.0, at).mul_(size.reshape(-1).square()).mul_(real)
        del size, grad
        if case["bits"] == 32:
            s["m"], s["v"] = m, v
        else:
            s["m"], s["m_scale"] = _held(m)
            s["v"], s["v_scale"] = _held(v.sqrt())
        if case["copy"]:
            s["copy"] = s["theta"].to(torch.bfloat16)
        s["where"], s["seed"] = where, int(seed) & 0xFFFFFFFF
        s["step"], s["lr"], s["beta1"], s["beta2"], s["eps"] = 100, 3e-4, 0.9, 0.999, 1e-8
        if own:                                # the optimiser's object, which a program makes once
            import paper_1907_10134_amd as bp
            cut = lambda flat, unit=1: [flat[o // unit:o // unit + -(-n // unit)] for o, n, _ in where]
            state = {"m": cut(s["m"]), "v": cut(s["v"])}
            if case["bits"] == 8:
                state.update(m_scale=cut(s["m_scale"], BLOCK), v_scale=cut(s["v_scale"], BLOCK))
            s["optimiser"] = bp.AdamW(cut(s["theta"]), cut(s["grad"]), state_bits=case["bits"], lr=s["lr"], beta1=s["beta1"],
                                      beta2=s["beta2"], eps=s["eps"], weight_decay=[w for _, _, w in where],
                                      copies=cut(s["copy"]) if case["copy"] else None, state=state)
        return s
    t, B, D = TYPES[case["type"]], case["B"], case["D"]
    if kind.endswith("token"):
        slots = torch.randperm(case["slots"], generator=g, device=DEV)[:B].to(torch.int32)
        if B > 4:
            slots[3] = -1                      # a row of the batch that no stream uses now
        s["slots"] = slots
        if kind == "conv_token":
            s["x"] = _normal(g, B, 2 * D).to(t)[:, :D]
            s["state"] = _normal(g, case["slots"], case["W"] - 1, D).to(t)
        else:
            N, G = case["N"], case["G"]
            s["A"], s["skip"], s["dt_bias"] = _layer(g, D, N)
            s["u"], s["dt"] = _normal(g, B, D).to(t), _normal(g, B, D).mul_(0.5).to(t)
            s["z"] = _normal(g, B, 2 * D).to(t)[:, D:] if case["z"] else None
            proj = _normal(g, B, 8 + 2 * G * N).to(t)
            s["Bm"], s["Cm"] = proj[:, 8:8 + G * N].unflatten(1, (G, N)), proj[:, 8 + G * N:].unflatten(1, (G, N))
            s["state"] = _normal(g, case["slots"], D, N)
            return s
    elif kind.startswith("conv"):
        s["x"] = _rows(g, case, 2 * D)[:, :, :D]
        s["state0"] = _normal(g, B, case["W"] - 1, D).to(t) if case["state0"] else None
        s["lengths"] = _lengths(g, case) if case["ragged"] else None
        if kind == "conv_train":
            s["dy"] = _rows(g, case, D)
    else:
        N, G = case["N"], case["G"]
        s["A"], s["skip"], s["dt_bias"] = _layer(g, D, N)
        s["u"], s["dt"] = _rows(g, case, D), _rows(g, case, D).mul_(0.5)
        s["z"] = _rows(g, case, 2 * D)[:, :, D:] if case["z"] else None
        proj = _rows(g, case, 8 + 2 * G * N)
        s["Bm"], s["Cm"] = proj[:, :, 8:8 + G * N].unflatten(2, (G, N)), proj[:, :, 8 + G * N:].unflatten(2, (G, N))
        s["h0"] = _normal(g, B, D, N) if case["h0"] else None
        s["lengths"] = _lengths(g, case) if case["ragged"] else None
        if kind == "scan_train":
            s["dy"] = _rows(g, case, D)
        return s
    bound = 1 / math.sqrt(case["W"])
    s["weight"], s["bias"] = _uniform(g, -bound, bound, D, case["W"]), _uniform(g, -bound, bound, D)
    return s


# ---- the operators in their plain form -----------------------------------------------------------

def _softplus(x):
    return x.clamp(min=0) + torch.log1p(torch.exp(-x.abs()))


def _sigmoid(x):
    e = torch.exp(-x.abs())
    return torch.where(x >= 0, 1 / (1 + e), e / (1 + e))


def _inside(s, T):
    """[T, B, 1] truth values: tokens of a sample; None where all are."""
    if s["lengths"] is None:
        return None
    return (torch.arange(T, device=DEV)[:, None] < s["lengths"][None])[..., None]


def _kept(x, inside):
    x = x.float()
    return x if inside is None else torch.where(inside, x, 0.0)


def _recur(a, b):
    """h[t] = a[t] h[t-1] + b[t] for all t by doubling the distance; a and b are used up, b becomes h."""
    k = 1
    while k < len(b):
        b[k:] += a[k:] * b[:-k]
        if 2 * k < len(b):
            a[k:] = a[k:] * a[:-k]
        k *= 2
    return b


def _recur_back(a, b):
    """g[t] = a[t + 1] g[t + 1] + b[t]; a[0] does not matter."""
    return _recur(torch.cat((a[:1], a[1:].flip(0))), b.flip(0)).flip(0)


def _scan_parts(s):
    """Inputs in 32 bits, channels as [G, D / G], with the steps, their decay and what enters the state."""
    G, T, B, D = s["Bm"].shape[2], *s["u"].shape
    inside = _inside(s, T)
    cut = lambda x: _kept(x, inside).unflatten(2, (G, D // G))
    narrow = inside if inside is None else inside[..., None]
    raw = _kept(s["dt"], inside) + s["dt_bias"]
    step = _softplus(raw)
    step = (step if inside is None else torch.where(inside, step, 0.0)).unflatten(2, (G, D // G))
    u, Bm, Cm = cut(s["u"]), _kept(s["Bm"], narrow), _kept(s["Cm"], narrow)
    A = s["A"].unflatten(0, (G, D // G))
    a = torch.exp(step[..., None] * A)
    b = (step * u)[..., None] * Bm[:, :, :, None]
    h0 = s["h0"].unflatten(1, (G, D // G)) if s["h0"] is not None else torch.zeros_like(b[0])
    b[0] += a[0] * h0
    return inside, cut, raw, step, u, Bm, Cm, A, a, b, h0


def _plain_scan(s, gradients):
    t = s["u"].dtype
    inside, cut, raw, step, u, Bm, Cm, A, a, b, h0 = _scan_parts(s)
    h = _recur(a.clone(), b)
    ungated = (h * Cm[:, :, :, None]).sum(-1) + s["skip"].unflatten(0, A.shape[:2]) * u
    out = lambda x, kind=t: _kept(x.flatten(2), inside).to(kind)
    z = cut(s["z"]) if s["z"] is not None else None
    y = ungated if z is None else ungated * (z * _sigmoid(z))
    r = {"y": out(y), "h_last": h[-1].flatten(1, 2)}
    if not gradients:
        return r
    del r["h_last"]
    dy = cut(s["dy"])
    q = dy
    if z is not None:
        sg = _sigmoid(z)
        r["dz"] = out(dy * ungated * sg * (1 + z * (1 - sg)))
        q = dy * z * sg
    g = _recur_back(a, q[..., None] * Cm[:, :, :, None])
    r["dCm"] = (h * q[..., None]).sum(3).to(t)
    r["dBm"] = (g * (step * u)[..., None]).sum(3).to(t)
    s1 = (g * Bm[:, :, :, None]).sum(-1)
    before = torch.cat((h0[None], h[:-1]))
    del h
    g *= a                                     # dL/dh of the state before, through the decay alone
    r["dh0"] = g[0].flatten(1, 2).clone()
    g *= before
    ds = u * s1 + (g * A).sum(-1)
    r["du"] = out(step * s1 + s["skip"].unflatten(0, A.shape[:2]) * q)
    ddt = _kept(ds.flatten(2) * _sigmoid(raw), inside)
    r["ddt"], r["ddt_bias"] = ddt.to(t), ddt.sum((0, 1))
    r["dA"] = (g * step[..., None]).sum((0, 1)).flatten(0, 1)
    r["dskip"] = (q * u).sum((0, 1)).flatten()
    return r


def _plain_scan_token(s):
    G, B, D = s["Bm"].shape[1], *s["u"].shape
    used = s["slots"] >= 0
    at = s["slots"].clamp(min=0).long()
    step = _softplus(s["dt"].float() + s["dt_bias"])
    u = s["u"].float()
    wide = lambda x: x.float().repeat_interleave(D // G, 1)
    h = torch.exp(step[..., None] * s["A"]) * s["state"][at] + (step * u)[..., None] * wide(s["Bm"])
    y = (h * wide(s["Cm"])).sum(-1) + s["skip"] * u
    if s["z"] is not None:
        z = s["z"].float()
        y = y * z * _sigmoid(z)
    s["state"][at[used]] = h[used]
    return {"y": torch.where(used[:, None], y, 0.0).to(s["u"].dtype), "state": s["state"]}


def _plain_conv(s, gradients):
    x, W = s["x"], s["weight"].shape[1]
    (T, B, D), t, w = x.shape, x.dtype, s["weight"]
    inside = _inside(s, T)
    before = s["state0"].transpose(0, 1).float() if s["state0"] is not None else torch.zeros((W - 1, B, D), device=DEV)
    xp = torch.cat((before, _kept(x, inside)))
    p = s["bias"] + sum(w[:, k] * xp[k:k + T] for k in range(W))
    silu = s["case"]["silu"]
    sg = _sigmoid(p) if silu else None
    y = _kept(p * sg if silu else p, inside).to(t)
    if not gradients:
        n = s["lengths"] if s["lengths"] is not None else torch.full((B,), T, device=DEV)
        at = n[None].long() + torch.arange(W - 1, device=DEV)[:, None]
        last = xp.gather(0, at[..., None].expand(W - 1, B, D))
        return {"y": y, "state_last": last.transpose(0, 1).to(t)}
    dp = _kept(s["dy"], inside)
    if silu:
        dp = dp * sg * (1 + p * (1 - sg))
    dxp = torch.zeros_like(xp)
    for k in range(W):
        dxp[k:k + T] += w[:, k] * dp
    dw = torch.stack([(dp * xp[k:k + T]).sum((0, 1)) for k in range(W)], 1)
    r = {"y": y, "dx": _kept(dxp[W - 1:], inside).to(t), "dweight": dw, "dbias": dp.sum((0, 1))}
    if s["state0"] is not None:
        r["dstate0"] = dxp[:W - 1].transpose(0, 1).to(t)
    return r


def _plain_conv_token(s):
    used = s["slots"] >= 0
    at = s["slots"].clamp(min=0).long()
    seen = torch.cat((s["state"][at], s["x"][:, None]), 1)         # [B, W, D]
    p = s["bias"] + (seen.float() * s["weight"].t()).sum(1)
    y = p * _sigmoid(p) if s["case"]["silu"] else p
    s["state"][at[used]] = seen[used, 1:]
    return {"y": torch.where(used[:, None], y, 0.0).to(s["x"].dtype), "state": s["state"]}


def _held(x, up=None):
    """(e4m3 values, scales) of x in blocks: the largest of a block stands at 448.  To the nearest, or, with `up` in
    [0, 1) for each value, down or up by chance; a value above zero does not become zero then."""
    x = x.reshape(-1, BLOCK)
    scale = x.abs().amax(1).clamp(min=2.0 ** -100) * (1 / 448)
    q = x * (1 / scale)[:, None]
    if up is not None:
        unit = torch.exp2(torch.floor(torch.log2(q.clamp(min=2.0 ** -6))) - 3)
        low = torch.floor(q / unit) * unit
        chosen = torch.where((q - low) / unit + up.reshape(q.shape) >= 1, low + unit, low)
        q = torch.where(q > 0, chosen.clamp(min=2.0 ** -9, max=448.0), q)
    return q.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).reshape(-1), scale


def _chance(s, n, tensor):
    """[0, 1) for each of n places of a tensor: two rounds of multiply and fold over the place, the tensor and the seed."""
    low = 0xFFFFFFFF
    first = (s["seed"] * 0x9E3779B1 + tensor * 0x6A09E667) & low
    x = (torch.arange(n, device=DEV, dtype=torch.int64) + first) & low
    for k in (0xBB67AE85, 0x3C6EF373):
        x = ((x ^ (x >> 16)) * k) & low
    x = x ^ (x >> 15)
    return (x >> 8).float() * 2.0 ** -24


def _plain_adamw(s):
    b1, b2, n, lr = s["beta1"], s["beta2"], s["step"], s["lr"]
    grad, eight = s["grad"].float(), s["case"]["bits"] == 8
    decay = torch.cat([torch.full((-(-k // BLOCK),), w, device=DEV) for _, k, w in s["where"]])
    if eight:
        m = (s["m"].float().reshape(-1, BLOCK) * s["m_scale"][:, None]).reshape(-1)
        v = (s["v"].float().reshape(-1, BLOCK) * s["v_scale"][:, None]).reshape(-1).square()
    else:
        m, v = s["m"], s["v"]
    m.mul_(b1).add_(grad, alpha=1 - b1)
    v.mul_(b2).addcmul_(grad, grad, value=1 - b2)
    root = v.sqrt()
    update = (m / (1 - b1 ** n)) / (root / math.sqrt(1 - b2 ** n) + s["eps"])
    theta = s["theta"].view(-1, BLOCK)
    theta.mul_(1 - lr * decay[:, None]).sub_(update.view(-1, BLOCK), alpha=lr)
    out = {"theta": s["theta"], "m": s["m"], "v": s["v"]}
    if s["case"]["copy"]:
        s["copy"].copy_(s["theta"])
        out["copy"] = s["copy"]
    if eight:
        up = torch.cat([_chance(s, -(-k // BLOCK) * BLOCK, i) for i, (_, k, _) in enumerate(s["where"])])
        for name, held in (("m", _held(m)), ("v", _held(root, up))):
            s[name].copy_(held[0])
            s[name + "_scale"].copy_(held[1])
            out[name + "_scale"] = s[name + "_scale"]
    return out


# ---- one pass ------------------------------------------------------------------------------------

def run(s):
    kind = s["kind"]
    if own:
        return _own(s)
    if kind == "adamw":
        return _plain_adamw(s)
    if kind == "scan_token":
        return _plain_scan_token(s)
    if kind == "conv_token":
        return _plain_conv_token(s)
    return (_plain_scan if kind.startswith("scan") else _plain_conv)(s, kind.endswith("train"))


def _own(s):
    import paper_1907_10134_amd as bp
    kind, case = s["kind"], s["case"]
    if kind == "adamw":
        s["optimiser"].t = s["step"] - 1
        s["optimiser"].step(seed=s["seed"])
        names = ["theta", "m", "v"] + ["copy"] * case["copy"] + ["m_scale", "v_scale"] * (case["bits"] == 8)
        return {k: s[k] for k in names}
    if kind == "scan_token":
        y = bp.ssm_scan_step(s["u"], s["dt"], s["A"], s["Bm"], s["Cm"], s["state"], skip=s["skip"], z=s["z"],
                             dt_bias=s["dt_bias"], slots=s["slots"])
        return {"y": y, "state": s["state"]}
    if kind == "conv_token":
        y = bp.ssm_conv_step(s["x"], s["weight"], s["bias"], s["state"], silu=case["silu"], slots=s["slots"])
        return {"y": y, "state": s["state"]}
    B, D = case["B"], case["D"]
    if kind.startswith("conv"):
        with_ = dict(silu=case["silu"], state0=s["state0"], lengths=s["lengths"])
        if kind == "conv_prompt":
            last = torch.empty((B, case["W"] - 1, D), dtype=s["x"].dtype, device=DEV)
            y = bp.ssm_conv(s["x"], s["weight"], s["bias"], state_last=last, **with_)
            return {"y": y, "state_last": last}
        d0 = torch.empty_like(s["state0"]) if s["state0"] is not None else None
        y = bp.ssm_conv(s["x"], s["weight"], s["bias"], **with_)
        g = bp.ssm_conv_backward(s["dy"], s["x"], s["weight"], s["bias"], dstate0=d0, **with_)
        r = {"y": y, "dx": g.dx, "dweight": g.dweight, "dbias": g.dbias}
        return dict(r, dstate0=d0) if d0 is not None else r
    inputs = (s["u"], s["dt"], s["A"], s["Bm"], s["Cm"])
    with_ = dict(skip=s["skip"], z=s["z"], dt_bias=s["dt_bias"], h0=s["h0"], lengths=s["lengths"])
    if kind == "scan_prompt":
        h_last = torch.empty((B, D, case["N"]), dtype=torch.float32, device=DEV)
        y = bp.ssm_scan(*inputs, h_last=h_last, **with_)
        return {"y": y, "h_last": h_last}
    states = bp.ssm_scan_states(*s["u"].shape, case["N"], device=DEV)
    dh0 = torch.empty((B, D, case["N"]), dtype=torch.float32, device=DEV)
    y = bp.ssm_scan(*inputs, states=states, **with_)
    g = bp.ssm_scan_backward(s["dy"], *inputs, states=states, dh0=dh0, **with_)
    r = {"y": y, "du": g.du, "ddt": g.ddt, "dA": g.dA, "dBm": g.dBm, "dCm": g.dCm, "dskip": g.dskip, "ddt_bias": g.ddt_bias,
         "dh0": dh0}
    return dict(r, dz=g.dz) if s["z"] is not None else r


# ---- what a pass cannot do without ---------------------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind == "adamw":
        n = sum(k for k, _ in _tensors(case))
        size = {"f32": 4, "bf16": 2, "f16": 2}[case["grad"]] + 8 + 2 * case["copy"]
        return {"bytes": n * (size + (16 if case["bits"] == 32 else 4 + 16 / BLOCK)), "flops": 14 * n}
    e = 4 if case["type"] == "f32" else 2
    B, D = case["B"], case["D"]
    if kind == "conv_token":
        return {"bytes": B * D * e * 2 * case["W"] + D * 4 * (case["W"] + 1), "flops": B * D * 2 * (case["W"] + 2)}
    if kind == "scan_token":
        N = case["N"]
        wide = B * e * (D * (3 + case["z"]) + 2 * case["G"] * N)
        return {"bytes": wide + 8 * B * D * N + 4 * D * (N + 2), "flops": 6 * B * D * N}
    rows = case["T"] * B                       # of the ragged ones about three quarters are read; all are written
    read = 0.75 * rows if case["ragged"] else rows
    if kind.startswith("conv"):
        W, train = case["W"], kind == "conv_train"
        return {"bytes": D * e * ((read + rows) + (2 * read + rows) * train) + 4 * D * (W + 1) * (1 + 2 * train),
                "flops": read * D * ((2 * W + 4) + (4 * W + 8) * train)}
    N, G, z = case["N"], case["G"], case["z"]
    bytes_ = e * (read * (D * (2 + z) + 2 * G * N) + rows * D) + 4 * D * (N + 2) + 4 * B * D * N * (1 + case["h0"])
    flops = 6 * read * D * N
    if kind == "scan_train":                   # backward: the inputs and dy again, their gradients once
        bytes_ += e * (read * (D * (3 + z) + 2 * G * N) + rows * (D * (2 + z) + 2 * G * N)) + 8 * D * (N + 2)
        flops += 18 * read * D * N
    return {"bytes": bytes_, "flops": flops}


# ---- the definitions in 64 bits, step by step ----------------------------------------------------

def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind == "adamw":
        return _exact_adamw(s)
    token = kind.endswith("token")
    if token:                                  # a sequence of one for each row that a stream uses
        rows = [i for i, k in enumerate(s["slots"].tolist()) if k >= 0]
        slots = s["slots"].long()[rows]
        lengths = [1] * len(rows)
        take = lambda x: None if x is None else x[rows].double()[None]
        names = ("x",) if kind == "conv_token" else ("u", "dt", "z", "Bm", "Cm")
        v = {k: take(s[k]) for k in names}
        first = s["state"][slots].double()
    else:
        if kind == "scan_train" and case["T"] * 60e-6 * 5 > 20:
            return None
        lengths = s["lengths"].tolist() if s["lengths"] is not None else [case["T"]] * case["B"]
        names = ("x",) if kind.startswith("conv") else ("u", "dt", "z", "Bm", "Cm")
        v = {k: None if s[k] is None else s[k].double() for k in names}
        first = s["state0" if kind.startswith("conv") else "h0"]
        if first is not None:
            first = first.double()
    if kind.startswith("conv"):
        y, last, grads = _exact_conv(s, v["x"], first, lengths, kind == "conv_train")
    else:
        y, last, grads = _exact_scan(s, v, first, lengths, kind == "scan_train")
    if token:
        whole, state = torch.zeros((case["B"], case["D"]), dtype=torch.float64, device=DEV), s["state"].double()
        whole[rows], state[slots] = y[0], last
        return {"y": whole, "state": state}
    if kind.endswith("train"):
        return dict(grads, y=y)
    return {"y": y, ("state_last" if kind.startswith("conv") else "h_last"): last}


def _leaf(x):
    return x.detach().clone().requires_grad_(True)


def _beyond(lengths, T):
    return torch.arange(T, device=DEV).view(T, 1, 1) >= torch.tensor(lengths, device=DEV).view(1, -1, 1)


def _exact_scan(s, v, h0, lengths, gradients):
    """The recurrence one token after the other; the gradients by differentiating it."""
    u, dt, z, Bm, Cm = (v[k] for k in ("u", "dt", "z", "Bm", "Cm"))
    (T, B, D), G, N = u.shape, Bm.shape[2], Bm.shape[3]
    off = _beyond(lengths, T)
    h0 = torch.zeros((B, D, N), dtype=torch.float64, device=DEV) if h0 is None else h0
    leaves = {"u": u, "dt": dt, "z": z, "Bm": Bm, "Cm": Cm, "A": s["A"].double(), "skip": s["skip"].double(),
              "dt_bias": s["dt_bias"].double(), "h0": h0}
    with torch.set_grad_enabled(gradients):
        if gradients:
            leaves = {k: None if x is None else _leaf(x) for k, x in leaves.items()}
        x, raw, A = leaves["u"], leaves["dt"] + leaves["dt_bias"], leaves["A"].view(G, D // G, N)
        size = torch.where(raw > 30, raw, torch.log1p(torch.exp(raw.clamp(max=30)))).masked_fill(off, 0.0)
        size, x = size.unbind(0), x.masked_fill(off, 0.0).unbind(0)
        into, out = (leaves[k].masked_fill(off[..., None], 0.0).unbind(0) for k in ("Bm", "Cm"))
        h, ys = leaves["h0"].view(B, G, D // G, N), []
        for t in range(T):
            d, w = size[t].view(B, G, -1, 1), x[t].view(B, G, -1, 1)
            h = torch.exp(d * A) * h + d * w * into[t].unsqueeze(2)
            ys.append((h * out[t].unsqueeze(2)).sum(3).view(B, D))
        y = torch.stack(ys) + leaves["skip"] * torch.stack(x)
        if z is not None:
            y = y * torch.nn.functional.silu(leaves["z"].masked_fill(off, 0.0))
        y = y.masked_fill(off, 0.0)
        if not gradients:
            return y, h.reshape(B, D, N), None
        of = [k for k, x in leaves.items() if x is not None]
        got = torch.autograd.grad(y, [leaves[k] for k in of], s["dy"].double().masked_fill(off, 0.0))
    return y.detach(), None, {"d" + k: g for k, g in zip(of, got)}


def _exact_conv(s, x, state0, lengths, gradients):
    """Every output as a product of its window with the taps; the gradients by differentiating it."""
    T, B, D = x.shape
    W = s["weight"].shape[1]
    off = _beyond(lengths, T)
    given = state0 is not None
    state0 = state0 if given else torch.zeros((B, W - 1, D), dtype=torch.float64, device=DEV)
    leaves = {"x": x, "state0": state0, "weight": s["weight"].double(), "bias": s["bias"].double()}
    with torch.set_grad_enabled(gradients):
        if gradients:
            leaves = {k: _leaf(a) for k, a in leaves.items()}
        row = torch.cat((leaves["state0"].transpose(0, 1), leaves["x"].masked_fill(off, 0.0)))
        p = (row.unfold(0, W, 1) * leaves["weight"]).sum(3) + leaves["bias"]
        y = (torch.nn.functional.silu(p) if s["case"]["silu"] else p).masked_fill(off, 0.0)
        if not gradients:
            return y, torch.stack([row[n:n + W - 1, i] for i, n in enumerate(lengths)]), None
        of = [k for k in leaves if given or k != "state0"]
        got = torch.autograd.grad(y, [leaves[k] for k in of], s["dy"].double().masked_fill(off, 0.0))
    return y.detach(), None, {"d" + k: g for k, g in zip(of, got)}


def _exact_adamw(s):
    """Tensor by tensor, every value from the formula; an 8-bit value by looking for its neighbours among all there are."""
    eight, t = s["case"]["bits"] == 8, s["step"]
    names = ["theta", "m", "v"] + ["copy"] * s["case"]["copy"] + ["m_scale", "v_scale"] * eight
    out = {k: torch.zeros(s[k].shape, dtype=torch.float64, device=DEV) for k in names}
    all_ = torch.arange(127, device=DEV, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    for i, (o, n, w) in enumerate(s["where"]):
        k = -(-n // BLOCK) * BLOCK
        here, blocks = slice(o, o + k), slice(o // BLOCK, (o + k) // BLOCK)
        m, v, g = s["m"][here].double(), s["v"][here].double(), s["grad"][here].double()
        if eight:
            m = (m.view(-1, BLOCK) * s["m_scale"][blocks].double()[:, None]).flatten()
            v = (v.view(-1, BLOCK) * s["v_scale"][blocks].double()[:, None]).flatten() ** 2
        m, v = s["beta1"] * m + (1 - s["beta1"]) * g, s["beta2"] * v + (1 - s["beta2"]) * g ** 2
        rate = (m / (1 - s["beta1"] ** t)) / ((v / (1 - s["beta2"] ** t)) ** 0.5 + s["eps"])
        theta = s["theta"][here].double()
        out["theta"][here] = theta - s["lr"] * (w * theta + rate)
        if s["case"]["copy"]:
            out["copy"][here] = out["theta"][here]
        if not eight:
            out["m"][here], out["v"][here] = m, v
            continue
        for name, x, by in (("m", m, None), ("v", v ** 0.5, _chance(s, k, i).double())):
            x = x.view(-1, BLOCK)
            scale = x.abs().max(1).values.clamp(min=2.0 ** -100) / 448
            q = (x / scale[:, None]).flatten()
            size = q.abs().clamp(max=448.0)
            above = torch.searchsorted(all_, size).clamp(1, 126)
            lo, hi = all_[above - 1], all_[above]
            share = (size - lo) / (hi - lo)
            if by is None:
                even = (above - 1) % 2 == 0
                value = torch.where((share < 0.5) | ((share == 0.5) & even), lo, hi)
            else:
                value = torch.where(share + by >= 1, hi, lo).clamp(min=2.0 ** -9)
                value = torch.where(size > 0, value, 0.0)
            out[name][here], out[name + "_scale"][blocks] = value * q.sign(), scale
    return out
