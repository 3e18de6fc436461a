"""A gated linear recurrence, the loss that trains a stack from a teacher's top logits, and the search that serves it with
beams, as cases that can be timed and compared.

Kinds, each a dict of plain values:

  gated_prompt  the gated recurrence over whole sequences, with the state after them: what serving does with a prompt.
  gated_train   the same forward and all its gradients: what a training step does with the layer.
  gated_token   one token of every running stream, the states held in slots of a cache and advanced in place.
  distil        the loss of a student against a teacher's top logits and its gradient for the student's logits.
  beam          one step of a beam search: selection over beams and vocabulary, and the move of the beams' states.

Activations and logits are float32, bfloat16 or float16; parameters, states and losses are float32.  Time comes first,
[T, B, channels], as everywhere in this package; `order` says how the memory lies ("tb": as the shape says, "bt": sequence
by sequence, the tensors are transposed views).  `ragged`: the samples have lengths of their own; what lies behind a sample's
end is padding of any value.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
MOST = 4 * 4096 * 4096                         # elements (T B D) of the largest recurrence
MOST_LOGITS = 8192 * 32768                     # of the largest loss
MOST_BEAMS = 64 * 8 * 131072                   # logits of the largest search
MOST_STATES = 64 * 8 * 4 * 2048                # beams times layers times channels there


def listed():
    return [
        # The smallest prompt of the package's configurations: nothing but latency.
        {"name": "gated_prompt_T16_B2_D40", "kind": "gated_prompt", "T": 16, "B": 2, "D": 40, "type": "f32", "z": False,
         "h0": False, "ragged": False, "order": "tb"},
        # A batch of ordinary prompts of different lengths, sequence by sequence in memory, an odd number of channels.
        {"name": "gated_prompt_T1000_B16_D641_f16", "kind": "gated_prompt", "T": 1000, "B": 16, "D": 641, "type": "f16",
         "z": True, "h0": False, "ragged": True, "order": "bt"},
        # One very long prompt that goes on from a state: all the parallelism there is lies along the sequence.
        {"name": "gated_prompt_T30000_B1_D2048_bf16", "kind": "gated_prompt", "T": 30000, "B": 1, "D": 2048, "type": "bf16",
         "z": True, "h0": True, "ragged": False, "order": "tb"},
        # Training in float32 with ragged lengths, as a piece of longer sequences: a state comes in, a gradient comes back.
        {"name": "gated_train_T1000_B16_D330_f32", "kind": "gated_train", "T": 1000, "B": 16, "D": 330, "type": "f32",
         "z": False, "h0": True, "ragged": True, "order": "tb"},
        # The training step of a large gated layer.
        {"name": "gated_train_T4096_B4_D4096_bf16", "kind": "gated_train", "T": 4096, "B": 4, "D": 4096, "type": "bf16",
         "z": True, "h0": False, "ragged": False, "order": "tb"},
        # One token of 64 running streams.
        {"name": "gated_token_B64_D4096_bf16", "kind": "gated_token", "B": 64, "D": 4096, "type": "bf16", "z": True,
         "slots": 80},
        # The loss of the package's own small stack: many short rows.
        {"name": "distil_T64_B32_V16_f32", "kind": "distil", "T": 64, "B": 32, "V": 16, "K": 8, "type": "f32",
         "temperature": 1.0, "tail": False, "hard": 0.0, "masked": False},
        # An ordinary batch with padding in it and an odd vocabulary, the teacher's other tokens as one more class.
        {"name": "distil_T1000_B16_V4001_f16", "kind": "distil", "T": 1000, "B": 16, "V": 4001, "K": 50, "type": "f16",
         "temperature": 1.0, "tail": True, "hard": 0.0, "masked": True},
        # A large batch and vocabulary, softened, with the data's own tokens for a part of the loss.
        {"name": "distil_T2048_B4_V32768_bf16", "kind": "distil", "T": 2048, "B": 4, "V": 32768, "K": 64, "type": "bf16",
         "temperature": 2.0, "tail": False, "hard": 0.3, "masked": False},
        # A search with the package's own small stack: nothing but latency.
        {"name": "beam_B2_W4_V16_f32", "kind": "beam", "B": 2, "W": 4, "V": 16, "type": "f32", "layers": 2, "D": 128},
        # One search over an ordinary vocabulary.
        {"name": "beam_B1_W5_V32001_bf16", "kind": "beam", "B": 1, "W": 5, "V": 32001, "type": "bf16", "layers": 8, "D": 1024},
        # Many searches over a large vocabulary, with some hundred megabytes of states.
        {"name": "beam_B64_W8_V131072_bf16", "kind": "beam", "B": 64, "W": 8, "V": 131072, "type": "bf16", "layers": 4,
         "D": 2048},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("gated_prompt", "gated_prompt", "gated_train", "gated_train", "gated_token", "distil", "distil", "distil",
                       "beam", "beam", "beam"))
    case = {"kind": kind, "type": rng.choice(("f32", "bf16", "bf16", "f16"))}
    if kind == "distil":
        case["V"] = _log_int(rng, 16, 131072)
        case["T"] = _log_int(rng, 1, min(4096, MOST_LOGITS // case["V"]))
        case["B"] = _log_int(rng, 1, max(1, min(64, MOST_LOGITS // (case["V"] * case["T"]))))
        return dict(case, K=_log_int(rng, 1, min(256, case["V"])), temperature=rng.choice((1.0, 1.0, 2.0, 0.7)),
                    tail=rng.random() < 0.4, hard=rng.choice((0.0, 0.0, 0.3, 1.0)), masked=rng.random() < 0.5)
    if kind == "beam":
        case["W"], case["V"] = _log_int(rng, 1, 32), _log_int(rng, 16, 131072)
        case["B"] = _log_int(rng, 1, min(128, MOST_BEAMS // (case["W"] * case["V"])))
        case["D"] = _log_int(rng, 16, 2048)
        room = MOST_STATES // (case["B"] * case["W"] * case["D"])
        return dict(case, layers=rng.randint(1, max(1, min(8, room))))
    if kind == "gated_token":
        case["B"], case["D"] = _log_int(rng, 1, 256), _log_int(rng, 64, 8192)
        return dict(case, slots=case["B"] + rng.randint(0, 32), z=rng.random() < 0.6)
    case["D"] = _log_int(rng, 16, 8192)
    case["T"] = _log_int(rng, 1, min(MOST // case["D"], 4096 if kind == "gated_train" else 30000))
    case["B"] = _log_int(rng, 1, max(1, min(64, MOST // (case["D"] * case["T"]))))
    return dict(case, z=rng.random() < 0.6, h0=rng.random() < 0.4, ragged=case["B"] > 1 and rng.random() < 0.4,
                order=rng.choice(("tb", "bt")))


# ---- inputs --------------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _normal(g, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=g, device=DEV, dtype=dtype)


def _uniform(g, lo, hi, *shape):
    return lo + (hi - lo) * torch.rand(shape, generator=g, device=DEV)


def _rows(g, case, width):
    """[T, B, width] normal values of the case's type, in its order."""
    T, B, t = case["T"], case["B"], TYPES[case["type"]]
    if case["order"] == "bt":
        return _normal(g, B, T, width, dtype=t).transpose(0, 1)
    return _normal(g, T, B, width, dtype=t)


def _lengths(g, case):
    """Half to all of T, and one sample that is empty and one of a single token."""
    T, B = case["T"], case["B"]
    n = torch.randint((T + 1) // 2, T + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
    n[-1] = 1
    if B > 2:
        n[1] = 0
    return n


def prepare(case, seed):
    g, kind = _gen(seed), case["kind"]
    s, t = {"case": case, "kind": kind}, TYPES[case["type"]]
    if kind == "distil":
        T, B, V, K = case["T"], case["B"], case["V"], case["K"]
        # a student on its way: its logits are the teacher's with as much of their own
        teacher = _normal(g, T * B, V).mul_(2.0)
        s["logits"] = torch.randn((T * B, V), generator=g, device=DEV).add_(teacher).to(t).view(T, B, V)
        teacher.mul_(1.5)
        top, index = teacher.topk(K, dim=-1)
        if K > 4:                              # the teacher's list ends early in some rows
            index[::3, K - K // 4:] = -1
        s["top_logits"], s["top_index"] = top.view(T, B, K), index.to(torch.int32).view(T, B, K)
        s["top_norm"] = None
        if case["tail"]:
            s["top_norm"] = torch.logsumexp(teacher.div_(case["temperature"]), -1).view(T, B)
        s["targets"] = None
        if case["hard"]:
            s["targets"] = torch.randint(0, V, (T, B), generator=g, device=DEV, dtype=torch.int32)
            s["targets"][:, 0][T // 2:] = -1   # a sample whose second half has no known tokens
        s["weight"] = None
        if case["masked"]:
            real = (torch.rand((T, B), generator=g, device=DEV) < 0.85).float()
            scale = 2.0 ** 14 if t is torch.float16 else 1.0       # gradients in float16 are kept off its subnormal range
            s["weight"] = real * (scale / real.sum().clamp(min=1))
        return s
    if kind == "beam":
        B, W, V, D = case["B"], case["W"], case["V"], case["D"]
        s["logits"] = _normal(g, B * W, V, dtype=t).mul_(2.5).view(B, W, V)
        s["scores"] = -_uniform(g, 1.0, 4.0, B, 1) - _uniform(g, 0.0, 3.0, B, W).sort(1).values
        s["finished"] = torch.rand((B, W), generator=g, device=DEV) < 0.1
        if B > 2:                              # a search that starts now: its beams are all the first one
            s["scores"][1, 1:] = -math.inf
            s["finished"][1] = False
        s["end"] = 2
        slots = B * W + 8
        s["slots"] = torch.randperm(slots, generator=g, device=DEV)[:B * W].to(torch.int32).view(B, W)
        s["states"] = []
        for _ in range(case["layers"]):        # of a stack of state space and gated layers, with their convolutions
            s["states"] += [_normal(g, slots, D, 16), _normal(g, slots, 3, D, dtype=torch.bfloat16), _normal(g, slots, D)]
        s["states"].append(torch.randint(0, V, (slots, 65), generator=g, device=DEV, dtype=torch.int32))
        if own:                                # the list of states, which a program makes once
            import paper_1907_10134_amd as bp
            s["mover"] = bp.BeamStates(s["states"])
        return s
    B, D = case["B"], case["D"]
    # decays such that a state lasts for some two to some two thousand tokens
    s["decay"] = torch.exp(_uniform(g, math.log(1e-3), 0.0, D))
    s["r_bias"], s["i_bias"] = _normal(g, D).mul_(0.5), _normal(g, D).mul_(0.5)
    if kind == "gated_token":
        slots = torch.randperm(case["slots"], generator=g, device=DEV)[:B].to(torch.int32)
        if B > 4:
            slots[3] = -1                      # a row of the batch that no stream uses now
        s["slots"] = slots
        s["x"] = _normal(g, B, D).to(t)
        s["z"] = _normal(g, B, 2 * D).to(t)[:, D:] if case["z"] else None
        gates = _normal(g, B, 2 * D).to(t)
        s["r"], s["i"] = gates[:, :D], gates[:, D:]
        s["state"] = _normal(g, case["slots"], D)
        return s
    s["x"] = _rows(g, case, D)
    gates = _rows(g, case, 2 * D)
    s["r"], s["i"] = gates[..., :D], gates[..., D:]
    s["z"] = _rows(g, case, 2 * D)[..., D:] if case["z"] else None
    s["h0"] = _normal(g, B, D) if case["h0"] else None
    s["lengths"] = _lengths(g, case) if case["ragged"] else None
    if kind == "gated_train":
        s["dy"] = _rows(g, case, D)
        s["dh_last"] = _normal(g, B, D) if case["h0"] else None
    return s


# ---- the operators in their plain form -----------------------------------------------------------

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


def _plain_gated(s, gradients):
    t, (T, B, D) = s["x"].dtype, s["x"].shape
    inside = _inside(s, T)
    out = lambda v: _kept(v, inside).to(t)
    x = _kept(s["x"], inside)
    rho, iota = _sigmoid(_kept(s["r"], inside) + s["r_bias"]), _sigmoid(_kept(s["i"], inside) + s["i_bias"])
    size = _kept(s["decay"] * rho, inside)     # behind an end the state stays as it is
    a, m = torch.exp(-size), torch.sqrt(-torch.expm1(-2 * size))
    b = m * iota * x
    h0 = s["h0"] if s["h0"] is not None else torch.zeros((B, D), device=DEV)
    b[0] += a[0] * h0
    h = _recur(a.clone(), b)
    z = _kept(s["z"], inside) if s["z"] is not None else None
    y = out(h if z is None else h * (z * _sigmoid(z)))
    if not gradients:
        return {"y": y, "h_last": h[-1].clone()}
    r, q = {"y": y}, _kept(s["dy"], inside)
    if z is not None:
        sg = _sigmoid(z)
        r["dz"] = out(q * h * sg * (1 + z * (1 - sg)))
        q = q * z * sg
    if s["dh_last"] is not None:
        q = q.clone()
        q[-1] += s["dh_last"]
    g = _recur_back(a, q)
    r["dh0"] = a[0] * g[0]
    r["dx"] = out(g * m * iota)
    di = _kept(g * m * x * iota * (1 - iota), inside)
    rate = _kept(g * a * (a * iota * x * (rho / m) - rho * torch.cat((h0[None], h[:-1]))), inside)
    dr = s["decay"] * (1 - rho) * rate
    r["dr"], r["di"] = dr.to(t), di.to(t)
    r["ddecay"], r["dr_bias"], r["di_bias"] = rate.sum((0, 1)), dr.sum((0, 1)), di.sum((0, 1))
    return r


def _plain_gated_token(s):
    used = s["slots"] >= 0
    at = s["slots"].clamp(min=0).long()
    rho, iota = _sigmoid(s["r"].float() + s["r_bias"]), _sigmoid(s["i"].float() + s["i_bias"])
    size = s["decay"] * rho
    h = torch.exp(-size) * s["state"][at] + torch.sqrt(-torch.expm1(-2 * size)) * iota * s["x"].float()
    y = h
    if s["z"] is not None:
        z = s["z"].float()
        y = h * z * _sigmoid(z)
    s["state"][at[used]] = h[used]
    return {"y": torch.where(used[:, None], y, 0.0).to(s["x"].dtype), "state": s["state"]}


def _softmax(x):
    """(shares, the logarithm of their sum before) along the last dimension."""
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(-1, keepdim=True)
    return e / total, top + torch.log(total)


def _plain_distil(s):
    case, V = s["case"], s["case"]["V"]
    tau, hard, kind = case["temperature"], case["hard"], s["logits"].dtype
    x = s["logits"].float().flatten(0, 1)
    index = s["top_index"].flatten(0, 1).long()
    here = index >= 0
    at = index.clamp(min=0)
    weight = torch.ones(len(x), device=DEV) if s["weight"] is None else s["weight"].flatten()
    q, norm = _softmax(x / tau)
    teacher = torch.where(here, s["top_logits"].flatten(0, 1).double() / tau, -math.inf)
    if s["top_norm"] is None:
        p = _softmax(teacher)[0]
    else:
        p = torch.exp(teacher - s["top_norm"].flatten()[:, None].double())
    logp = torch.where(p > 0, torch.log(p), 0.0)
    soft = (p * (logp - torch.where(here, x.gather(1, at) / tau - norm, 0.0))).sum(1)
    spread = torch.zeros((len(x), V + 1), device=DEV).scatter_add_(1, torch.where(here, at, V), p.float())[:, :V]
    if s["top_norm"] is None:
        d = q - spread
    else:
        p0 = (1 - p.sum(1)).clamp(min=0)
        inside = torch.zeros((len(x), V + 1), dtype=torch.bool, device=DEV).scatter_(1, torch.where(here, at, V), True)[:, :V]
        q0 = torch.where(inside, 0.0, q).sum(1)
        on = q0 > 0
        soft = soft + torch.where(on & (p0 > 0), p0 * torch.log(p0.clamp(min=1e-300) / torch.where(on, q0, 1.0)), 0.0)
        ratio = torch.where(on, p0 / torch.where(on, q0, 1.0), 1.0).float()
        d = torch.where(inside, q - spread, q * (1 - ratio)[:, None])
    loss, d = (1 - hard) * tau * tau * soft, d.mul_((1 - hard) * tau)
    if hard:
        target = s["targets"].flatten().long()
        known = target >= 0
        to = target.clamp(min=0)[:, None]
        q, norm = _softmax(x)
        loss = loss + hard * torch.where(known, (norm - x.gather(1, to))[:, 0], 0.0)
        q.scatter_add_(1, to, torch.full((len(x), 1), -1.0, device=DEV))
        d = d + hard * torch.where(known[:, None], q, 0.0)
    return {"loss": (weight * loss).float().view(s["logits"].shape[:2]), "dlogits": (weight[:, None] * d).to(kind).view(s["logits"].shape)}


def _plain_beam(s):
    (B, W, V), scores = s["logits"].shape, s["scores"].double()
    x = s["logits"].double()                   # sums of different beams can lie next to each other
    top = x.amax(-1, keepdim=True)
    logp = x - (top + torch.log(torch.exp(x - top).sum(-1, keepdim=True)))
    at_end = torch.arange(V, device=DEV) == s["end"]
    logp = torch.where(s["finished"][..., None], torch.where(at_end, 0.0, -math.inf), logp)
    order = (scores[..., None] + logp).view(B, W * V).sort(dim=1, descending=True, stable=True)
    total, flat = order.values[:, :W], order.indices[:, :W]
    parents, tokens = flat // V, flat % V
    # the first child of a beam goes on in its slot, the others take those of beams without one, in order
    same = (parents[:, :, None] == parents[:, None, :]) & torch.ones((W, W), dtype=torch.bool, device=DEV).tril(-1)
    more = same.any(2)
    childless = (parents[:, None, :] != torch.arange(W, device=DEV)[None, :, None]).all(2)
    free = torch.sort((~childless).int(), dim=1, stable=True).indices
    home = s["slots"].gather(1, parents)
    slots = torch.where(more, s["slots"].gather(1, free).gather(1, (more.cumsum(1) - 1).clamp(min=0)), home)
    sources = torch.where(more, home, -1)
    to, of = slots[more].long(), home[more].long()
    for state in s["states"]:
        state[to] = state[of]
    return {"scores": total.float(), "parents": parents.int(), "tokens": tokens.int(),
            "finished": s["finished"].gather(1, parents) | (tokens == s["end"]), "slots": slots, "sources": sources,
            "states": s["states"]}


# ---- one pass ------------------------------------------------------------------------------------

def run(s):
    kind = s["kind"]
    if own:
        return _own(s)
    if kind == "distil":
        return _plain_distil(s)
    if kind == "beam":
        return _plain_beam(s)
    if kind == "gated_token":
        return _plain_gated_token(s)
    return _plain_gated(s, kind == "gated_train")


def _own(s):
    import paper_1907_10134_amd as bp
    kind, case = s["kind"], s["case"]
    if kind == "distil":
        r = bp.distil(s["logits"], s["top_logits"], s["top_index"], temperature=case["temperature"], top_norm=s["top_norm"],
                      targets=s["targets"], hard=case["hard"], weight=s["weight"], gradient=True)
        return {"loss": r.loss, "dlogits": r.dlogits}
    if kind == "beam":
        c = bp.beam_select(s["logits"], s["scores"], finished=s["finished"], end=s["end"], slots=s["slots"])
        s["mover"].move(c.sources, c.slots)
        return {"scores": c.scores, "parents": c.parents, "tokens": c.tokens, "finished": c.finished, "slots": c.slots,
                "sources": c.sources, "states": s["states"]}
    inputs = (s["x"], s["r"], s["i"], s["decay"])
    with_ = dict(z=s["z"], r_bias=s["r_bias"], i_bias=s["i_bias"])
    if kind == "gated_token":
        return {"y": bp.gated_scan_step(*inputs, s["state"], slots=s["slots"], **with_), "state": s["state"]}
    T, B, D = s["x"].shape
    with_.update(h0=s["h0"], lengths=s["lengths"])
    if kind == "gated_prompt":
        h_last = torch.empty((B, D), dtype=torch.float32, device=DEV)
        return {"y": bp.gated_scan(*inputs, h_last=h_last, **with_), "h_last": h_last}
    states = bp.gated_scan_states(T, B, D, device=DEV)
    dh0 = torch.empty((B, D), dtype=torch.float32, device=DEV)
    y = bp.gated_scan(*inputs, states=states, **with_)
    g = bp.gated_scan_backward(s["dy"], *inputs, states, dh_last=s["dh_last"], dh0=dh0, **with_)
    r = {"y": y, "dh0": dh0, "dx": g.dx, "dr": g.dr, "di": g.di, "ddecay": g.ddecay, "dr_bias": g.dr_bias, "di_bias": g.di_bias}
    return dict(r, dz=g.dz) if s["z"] is not None else r


# ---- what a pass cannot do without ---------------------------------------------------------------

def work(case):
    kind, e = case["kind"], 4 if case["type"] == "f32" else 2
    if kind == "distil":
        rows, V, K = case["T"] * case["B"], case["V"], case["K"]
        read = 0.85 * rows if case["masked"] else rows
        exps = (2 if case["hard"] and case["temperature"] != 1 else 1)
        return {"bytes": read * (V * e + K * 8) + rows * (V * e + 8), "flops": read * V * (6 * exps + 2)}
    if kind == "beam":
        B, W, V, D = case["B"], case["W"], case["V"], case["D"]
        moved = sum((1 - 1 / W) ** W for _ in range(W)) * B        # children beyond the first, had each beam the same chance
        each = case["layers"] * (D * 64 + D * 6 + D * 4) + 260
        return {"bytes": 0.9 * B * W * V * e + B * W * 30 + 2 * moved * each, "flops": 4 * B * W * V}
    B, D, z = case["B"], case["D"], case["z"]
    if kind == "gated_token":
        return {"bytes": B * D * (e * (4 + z) + 8) + 12 * D, "flops": 24 * B * D}
    rows = case["T"] * B                       # of the ragged ones about three quarters are read; all are written
    read = 0.75 * rows if case["ragged"] else rows
    bytes_, flops = D * (e * (read * (3 + z) + rows) + 12 + 4 * B * (1 + case["h0"])), 24 * read * D
    if kind == "gated_train":                  # backward: the inputs and dy again, their gradients once
        bytes_ += D * (e * (read * (4 + z) + rows * (3 + z)) + 24 + 4 * B * (1 + 2 * case["h0"]))
        flops += 56 * read * D
    return {"bytes": bytes_, "flops": flops}


# ---- the definitions in 64 bits ------------------------------------------------------------------

def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind == "distil":
        return _exact_distil(s)
    if kind == "beam":
        return _exact_beam(s)
    if kind == "gated_token":                  # a sequence of one for each row that a stream uses
        rows = [i for i, k in enumerate(s["slots"].tolist()) if k >= 0]
        slots = s["slots"].long()[rows]
        take = lambda x: None if x is None else x[rows].double()[None]
        y, last, _ = _exact_gated(s, {k: take(s[k]) for k in ("x", "r", "i", "z")}, s["state"][slots].double(), [1] * len(rows), False)
        whole, state = torch.zeros((case["B"], case["D"]), dtype=torch.float64, device=DEV), s["state"].double()
        whole[rows], state[slots] = y[0], last
        return {"y": whole, "state": state}
    train = kind == "gated_train"
    lengths = s["lengths"].tolist() if s["lengths"] is not None else [case["T"]] * case["B"]
    h0 = torch.zeros((case["B"], case["D"]), dtype=torch.float64, device=DEV) if s["h0"] is None else s["h0"].double()
    v = {k: None if s[k] is None else s[k].double() for k in ("x", "r", "i", "z")}
    y, last, grads = _exact_gated(s, v, h0, lengths, train)
    return dict(grads, y=y) if train else {"y": y, "h_last": last}


def _exact_gated(s, v, h0, lengths, gradients):
    """The recurrence one token after the other; the gradients by differentiating it."""
    T, B, _ = v["x"].shape
    off = torch.arange(T, device=DEV).view(T, 1, 1) >= torch.tensor(lengths, device=DEV).view(1, -1, 1)
    leaves = {k: x if x is None else x.masked_fill(off, 0.0) for k, x in v.items()}
    leaves.update({k: s[k].double() for k in ("decay", "r_bias", "i_bias")}, h0=h0)
    if gradients:
        leaves = {k: None if x is None else x.detach().clone().requires_grad_(True) for k, x in leaves.items()}
    with torch.set_grad_enabled(gradients):
        size = leaves["decay"] * torch.sigmoid(leaves["r"] + leaves["r_bias"])
        into = (-torch.expm1(-2 * size)) ** 0.5 * torch.sigmoid(leaves["i"] + leaves["i_bias"]) * leaves["x"]
        decays, into = torch.exp(-size).masked_fill(off, 1.0).unbind(0), into.masked_fill(off, 0.0).unbind(0)
        h, hs = leaves["h0"], []
        for a, b in zip(decays, into):
            h = a * h + b
            hs.append(h)
        y = torch.stack(hs)
        if v["z"] is not None:
            y = y * torch.nn.functional.silu(leaves["z"])
        y = y.masked_fill(off, 0.0)
        if not gradients:
            return y, h, None
        of = [k for k, x in leaves.items() if x is not None]
        dlast = torch.zeros_like(h) if s["dh_last"] is None else s["dh_last"].double()
        got = torch.autograd.grad([y, h], [leaves[k] for k in of], [s["dy"].double().masked_fill(off, 0.0), dlast])
    return y.detach(), None, {"d" + k: g for k, g in zip(of, got)}


def _exact_distil(s):
    """The loss a few samples at a time; the gradient by differentiating it."""
    case, V = s["case"], s["case"]["V"]
    tau, hard = case["temperature"], case["hard"]
    losses, grads, T = [], [], case["T"]
    step = max(1, (1 << 25) // (V * case["B"]))
    for t in range(0, T, step):
        x = s["logits"][t:t + step].double().requires_grad_(True)
        index = s["top_index"][t:t + step].long()
        here = index >= 0
        teacher = (s["top_logits"][t:t + step].double() / tau).masked_fill(~here, -math.inf)
        logq = torch.log_softmax(x / tau, -1)
        if case["tail"]:
            logp = teacher - s["top_norm"][t:t + step].double()[..., None]
        else:
            logp = torch.log_softmax(teacher, -1)
        p = torch.exp(logp)
        of = logq.gather(-1, index.clamp(min=0))
        loss = (p * (logp - of).masked_fill(~here, 0.0)).sum(-1)
        if case["tail"]:
            inside = torch.zeros(x.shape[:2] + (V + 1,), dtype=torch.bool, device=DEV)
            inside.scatter_(-1, index.masked_fill(~here, V), True)
            rest = torch.logsumexp(logq.masked_fill(inside[..., :V], -math.inf), -1)
            p0, on = (1 - p.sum(-1)).clamp(min=0), ~inside[..., :V].all(-1)
            loss = loss + torch.where(on & (p0 > 0), p0 * (torch.log(p0.clamp(min=1e-300)) - rest.masked_fill(~on, 0.0)), 0.0)
        loss = (1 - hard) * tau * tau * loss
        if hard:
            target = s["targets"][t:t + step].long()
            ce = -torch.log_softmax(x, -1).gather(-1, target.clamp(min=0)[..., None])[..., 0]
            loss = loss + hard * ce.masked_fill(target < 0, 0.0)
        if s["weight"] is not None:
            loss = loss * s["weight"][t:t + step].double()
        grads.append(torch.autograd.grad(loss.sum(), x)[0])
        losses.append(loss.detach())
    return {"loss": torch.cat(losses), "dlogits": torch.cat(grads)}


def _exact_beam(s):
    """Beam by beam and sequence by sequence; the whole values are the selection's own and have no value in 64 bits."""
    (B, W, V), k = s["logits"].shape, min(s["case"]["W"], s["case"]["V"])
    scores = torch.empty((B, W), dtype=torch.float64, device=DEV)
    parents = []
    for b in range(B):
        found = []
        for w in range(W):
            start = float(s["scores"][b, w])
            if bool(s["finished"][b, w]):
                found.append((start, w))
                continue
            logp = torch.log_softmax(s["logits"][b, w].double(), -1).topk(k).values
            found += [(start + v, w) for v in logp.tolist()]
        found.sort(key=lambda f: (-f[0], f[1]))
        scores[b] = torch.tensor([f[0] for f in found[:W]], dtype=torch.float64)
        parents.append([f[1] for f in found[:W]])
    slots, to, of = s["slots"].tolist(), [], []
    for b in range(B):
        free = [w for w in range(W) if w not in parents[b]]
        seen = set()
        for p in parents[b]:
            if p in seen:
                to.append(slots[b][free.pop(0)]), of.append(slots[b][p])
            seen.add(p)
    states = []
    for state in s["states"]:
        if not state.is_floating_point():
            states.append(None)
            continue
        new = state.double()
        for i, j in zip(to, of):
            new[i] = state[j].double()
        states.append(new)
    return {"scores": scores, "parents": None, "tokens": None, "finished": None, "slots": None, "sources": None, "states": states}
