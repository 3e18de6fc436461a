"""A small stack of selective state space layers, trained and served with the library's operators.

A layer: root-mean-square norm, a projection to two halves, the short convolution and the selective scan of the first half
gated by the second, a projection back that is added to the stream.  A gated layer has the gated linear recurrence in the
scan's place, whose two gates come out of one projection.  The projections, norms and the loss on tokens are plain torch;
the convolution, the recurrences, their gradients, their single-token steps, the loss against another stack's top logits, the
selection of a beam search with the move of its states and the optimiser are the library's.  Activations are bfloat16, the
stream between the layers and all parameters float32; the projections use the bfloat16 copies that the optimiser keeps.

    python -m workloads.ssm_stack        trains on sequences with a delayed rule, continues some token by token, and lets a
                                         smaller stack with a gated layer learn from the first one's top logits
"""
from __future__ import annotations

import math

import torch

import paper_1907_10134_amd as bp

BF16 = torch.bfloat16
DECAYED = ("embed", "in_proj", "x_proj", "dt_proj", "gate_proj", "out_proj")


def _norm(x, weight):
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)
    return x * r * weight, r


def _norm_backward(g, x, r, weight):
    """(dx, dweight) of _norm."""
    n = x * r
    gw = g * weight
    return r * (gw - n * (gw * n).mean(-1, keepdim=True)), (g * n).flatten(0, -2).sum(0)


def _mm(x, w):
    """x @ w.T over all leading dimensions, as one product of two matrices."""
    return torch.mm(x.flatten(0, -2), w.t()).unflatten(0, x.shape[:-1])


class SsmStack:
    def __init__(self, vocabulary=16, width=64, layers=2, states=16, taps=4, state_bits=8, lr=3e-3, seed=0, device="cuda",
                 gated=()):
        """gated: the numbers of the layers that have the gated linear recurrence."""
        gen = torch.Generator().manual_seed(seed)
        normal = lambda scale, *shape: torch.randn(shape, generator=gen) * scale
        uniform = lambda lo, hi, *shape: lo + (hi - lo) * torch.rand(shape, generator=gen)
        d, D, N, R = width, 2 * width, states, -(-width // 16)
        self.sizes, self.layers, self.taps, self.gated = (d, D, N, R), layers, taps, frozenset(gated)
        p = {"embed": normal(0.3, vocabulary, d), "last_norm": torch.ones(d)}
        for l in range(layers):
            if l in self.gated:                # decays of 0.002 to 0.7: gates of one half remember one to 1000 steps
                p.update({"norm%d" % l: torch.ones(d), "in_proj%d" % l: normal(d ** -0.5, 2 * D, d),
                          "conv_w%d" % l: uniform(-0.5, 0.5, D, taps), "conv_b%d" % l: torch.zeros(D),
                          "gate_proj%d" % l: normal(D ** -0.5, 2 * D, D), "r_bias%d" % l: torch.zeros(D),
                          "i_bias%d" % l: torch.zeros(D), "decay_log%d" % l: uniform(math.log(2e-3), math.log(0.7), D),
                          "out_proj%d" % l: normal(D ** -0.5, d, D)})
                continue
            step = torch.exp(uniform(math.log(1e-3), math.log(0.1), D))
            p.update({"norm%d" % l: torch.ones(d), "in_proj%d" % l: normal(d ** -0.5, 2 * D, d),
                      "conv_w%d" % l: uniform(-0.5, 0.5, D, taps), "conv_b%d" % l: torch.zeros(D),
                      "x_proj%d" % l: normal(D ** -0.5, R + 2 * N, D), "dt_proj%d" % l: normal(R ** -0.5, D, R),
                      "dt_bias%d" % l: step + torch.log(-torch.expm1(-step)),
                      "A_log%d" % l: torch.log(torch.arange(1, N + 1).float()).expand(D, N).contiguous(),
                      "skip%d" % l: torch.ones(D), "out_proj%d" % l: normal(D ** -0.5, d, D)})
        self.p = {k: v.to(device) for k, v in p.items()}
        self.g = {k: torch.zeros_like(v) for k, v in self.p.items()}
        self.w = {k: v.to(BF16) for k, v in self.p.items()}
        self.optimiser = bp.AdamW(self.p.values(), self.g.values(), state_bits=state_bits, lr=lr, copies=list(self.w.values()),
                                  weight_decay=[0.1 if k.rstrip("0123456789") in DECAYED else 0.0 for k in self.p])

    def _cut(self, proj):
        """The step's low-rank part, Bm and Cm out of one projection."""
        N, R = self.sizes[2:]
        return proj[..., :R], proj[..., R:R + N].unflatten(-1, (1, N)), proj[..., R + N:].unflatten(-1, (1, N))

    def forward(self, tokens, lengths=None, keep=None, caches=None):
        """Logits [T, B, vocabulary] of tokens [T, B].  keep: a list that receives what backward() reads.  caches: (scan
        states [B, D, N], of a gated layer [B, D], last inputs [B, taps - 1, D]) of each layer, filled with the state after each
        sample."""
        p, w = self.p, self.w
        D = self.sizes[1]
        T, B = tokens.shape
        x = p["embed"][tokens]
        for l in range(self.layers):
            n, r = _norm(x, p["norm%d" % l])
            n = n.to(BF16)
            xz = _mm(n, w["in_proj%d" % l])
            u, z = xz[..., :D], xz[..., D:]
            h_last, last = caches[l] if caches is not None else (None, None)
            c = bp.ssm_conv(u, p["conv_w%d" % l], p["conv_b%d" % l], lengths=lengths, state_last=last)
            if l in self.gated:
                gates, decay = _mm(c, w["gate_proj%d" % l]), torch.exp(p["decay_log%d" % l])
                states = bp.gated_scan_states(T, B, D, device=x.device) if keep is not None else None
                y = bp.gated_scan(c, gates[..., :D], gates[..., D:], decay, z=z, r_bias=p["r_bias%d" % l], i_bias=p["i_bias%d" % l],
                                  lengths=lengths, h_last=h_last, states=states)
                if keep is not None:
                    keep.append((x, r, n, u, z, c, gates, decay, states, y))
                x = x + _mm(y, w["out_proj%d" % l]).float()
                continue
            proj = _mm(c, w["x_proj%d" % l])
            low, Bm, Cm = self._cut(proj)
            dt = _mm(low, w["dt_proj%d" % l])
            A = -torch.exp(p["A_log%d" % l])
            states = bp.ssm_scan_states(T, B, *self.sizes[1:3], device=x.device) if keep is not None else None
            y = bp.ssm_scan(c, dt, A, Bm, Cm, skip=p["skip%d" % l], z=z, dt_bias=p["dt_bias%d" % l], lengths=lengths,
                            h_last=h_last, states=states)
            if keep is not None:
                keep.append((x, r, n, u, z, c, low, Bm, Cm, dt, A, states, y))
            x = x + _mm(y, w["out_proj%d" % l]).float()
        n, r = _norm(x, p["last_norm"])
        n = n.to(BF16)
        if keep is not None:
            keep.append((x, r, n))
        return _mm(n, w["embed"]).float()

    def train_step(self, tokens, targets, lengths=None):
        """One iteration on tokens and targets [T, B]; the mean loss over the real tokens, before the update."""
        keep = []
        T, B = tokens.shape
        logits = self.forward(tokens, lengths, keep)
        logp = torch.log_softmax(logits, -1)
        real = self._real(T, B, lengths)
        loss = -(logp.gather(-1, targets[..., None])[..., 0] * real).sum()
        dlogits = torch.exp(logp)
        dlogits.scatter_add_(-1, targets[..., None], torch.full((T, B, 1), -1.0, device=logits.device))
        self._backward((dlogits * real[..., None]).to(BF16), tokens, lengths, keep)
        return loss

    def distil_step(self, tokens, top_logits, top_index, lengths=None, **how):
        """One iteration on tokens [T, B] against a teacher's top logits and their indices [T, B, K]; the mean loss over the real
        tokens, before the update.  how: what bp.distil takes besides."""
        keep = []
        T, B = tokens.shape
        logits = self.forward(tokens, lengths, keep)
        made = bp.distil(logits, top_logits, top_index, weight=self._real(T, B, lengths), dlogits=logits, **how)
        self._backward(made.dlogits.to(BF16), tokens, lengths, keep)
        return made.loss.sum()

    def _real(self, T, B, lengths):
        """[T, B]: each real token's share of them all."""
        device = self.p["embed"].device
        real = torch.ones((T, B), device=device) if lengths is None else (torch.arange(T, device=device)[:, None] < lengths).float()
        return real / real.sum()

    def _backward(self, dlogits, tokens, lengths, keep):
        """The gradients behind those of the logits, and the update."""
        p, w, g = self.p, self.w, self.g
        D = self.sizes[1]
        outer = lambda a, b: torch.mm(a.flatten(0, -2).t(), b.flatten(0, -2)).float()        # sum over tokens of a b^T
        back = lambda a, weight: torch.mm(a.flatten(0, -2), weight).unflatten(0, a.shape[:-1])
        x, r, n = keep.pop()
        dembed = outer(dlogits, n)
        dx, dw = _norm_backward(back(dlogits, w["embed"]).float(), x, r, p["last_norm"])
        g["last_norm"].copy_(dw)
        for l in reversed(range(self.layers)):
            if l in self.gated:
                x, r, n, u, z, c, gates, decay, states, y = keep.pop()
                out = dx.to(BF16)
                g["out_proj%d" % l].copy_(outer(out, y))
                s = bp.gated_scan_backward(back(out, w["out_proj%d" % l]), c, gates[..., :D], gates[..., D:], decay, states, z=z,
                                           r_bias=p["r_bias%d" % l], i_bias=p["i_bias%d" % l], lengths=lengths)
                g["decay_log%d" % l].copy_(s.ddecay * decay)
                g["r_bias%d" % l].copy_(s.dr_bias)
                g["i_bias%d" % l].copy_(s.di_bias)
                dgates = torch.cat((s.dr, s.di), -1)
                g["gate_proj%d" % l].copy_(outer(dgates, c))
                dc = s.dx + back(dgates, w["gate_proj%d" % l])
                dx = dx + self._front_backward(l, dc, s.dz, x, r, n, u, lengths, outer, back)
                continue
            x, r, n, u, z, c, low, Bm, Cm, dt, A, states, y = keep.pop()
            out = dx.to(BF16)
            g["out_proj%d" % l].copy_(outer(out, y))
            s = bp.ssm_scan_backward(back(out, w["out_proj%d" % l]), c, dt, A, Bm, Cm, states, skip=p["skip%d" % l], z=z,
                                     dt_bias=p["dt_bias%d" % l], lengths=lengths)
            g["A_log%d" % l].copy_(s.dA * A)
            g["skip%d" % l].copy_(s.dskip)
            g["dt_bias%d" % l].copy_(s.ddt_bias)
            g["dt_proj%d" % l].copy_(outer(s.ddt, low))
            dproj = torch.cat((back(s.ddt, w["dt_proj%d" % l]), s.dBm.flatten(2), s.dCm.flatten(2)), -1)
            g["x_proj%d" % l].copy_(outer(dproj, c))
            dc = s.du + back(dproj, w["x_proj%d" % l])
            dx = dx + self._front_backward(l, dc, s.dz, x, r, n, u, lengths, outer, back)
        g["embed"].copy_(dembed.index_add_(0, tokens.flatten(), dx.flatten(0, 1)))
        self.optimiser.step()

    def _front_backward(self, l, dc, dz, x, r, n, u, lengths, outer, back):
        """The gradient for the stream through what a layer has in front of its recurrence."""
        p, w, g = self.p, self.w, self.g
        k = bp.ssm_conv_backward(dc, u, p["conv_w%d" % l], p["conv_b%d" % l], lengths=lengths)
        g["conv_w%d" % l].copy_(k.dweight)
        g["conv_b%d" % l].copy_(k.dbias)
        dxz = torch.cat((k.dx, dz), -1)
        g["in_proj%d" % l].copy_(outer(dxz, n))
        dn, dw = _norm_backward(back(dxz, w["in_proj%d" % l]).float(), x, r, p["norm%d" % l])
        g["norm%d" % l].copy_(dw)
        return dn

    def caches(self, slots, device="cuda"):
        """Empty states of `slots` streams: (scan [slots, D, N] float32, of a gated layer [slots, D], convolution
        [slots, taps - 1, D]) of each layer."""
        _, D, N, _ = self.sizes
        return [(torch.zeros((slots, D) if l in self.gated else (slots, D, N), device=device),
                 torch.zeros((slots, self.taps - 1, D), dtype=BF16, device=device)) for l in range(self.layers)]

    def token(self, tokens, caches, slots=None):
        """Logits [B, vocabulary] behind one more token [B] of the streams in `slots`, whose states move on."""
        p, w = self.p, self.w
        D = self.sizes[1]
        x = p["embed"][tokens]
        for l in range(self.layers):
            h, last = caches[l]
            xz = _mm(_norm(x, p["norm%d" % l])[0].to(BF16), w["in_proj%d" % l])
            c = bp.ssm_conv_step(xz[:, :D], p["conv_w%d" % l], p["conv_b%d" % l], last, slots=slots)
            if l in self.gated:
                gates = _mm(c, w["gate_proj%d" % l])
                y = bp.gated_scan_step(c, gates[:, :D], gates[:, D:], torch.exp(p["decay_log%d" % l]), h, z=xz[:, D:],
                                       r_bias=p["r_bias%d" % l], i_bias=p["i_bias%d" % l], slots=slots)
                x = x + _mm(y, w["out_proj%d" % l]).float()
                continue
            low, Bm, Cm = self._cut(_mm(c, w["x_proj%d" % l]))
            y = bp.ssm_scan_step(c, _mm(low, w["dt_proj%d" % l]), -torch.exp(p["A_log%d" % l]), Bm, Cm, h,
                                 skip=p["skip%d" % l], z=xz[:, D:], dt_bias=p["dt_bias%d" % l], slots=slots)
            x = x + _mm(y, w["out_proj%d" % l]).float()
        return _mm(_norm(x, p["last_norm"])[0].to(BF16), w["embed"]).float()


    def beams(self, tokens, width, steps, lengths=None, end=-1):
        """The `width` best continuations of each prompt [T, B], of a token at least, that a beam search finds: (tokens
        [B, width, steps], scores [B, width]), best first.  What comes behind an `end` is `end`."""
        T, B = tokens.shape
        device = tokens.device
        prompt, caches = self.caches(B, device), self.caches(B * width, device)
        logits = self.forward(tokens, lengths, caches=prompt)
        last = torch.full((B,), T - 1, device=device) if lengths is None else (lengths - 1).long()
        logits = logits[last, torch.arange(B, device=device)]
        slots = torch.arange(B * width, dtype=torch.int32, device=device).view(B, width)
        for have, cache in zip(prompt, caches):
            for a, b in zip(have, cache):
                b[::width] = a                 # the first beam of each search; the others do not count yet
        scores = torch.full((B, width), -math.inf, device=device)
        scores[:, 0] = 0.0
        finished = torch.zeros((B, width), dtype=torch.bool, device=device) if end >= 0 else None
        history = torch.zeros((B * width, steps), dtype=torch.int32, device=device)
        states = bp.BeamStates([x for cache in caches for x in cache] + [history])
        logits = logits[:, None].expand(B, width, -1).contiguous()
        for k in range(steps):
            c = bp.beam_select(logits, scores, finished=finished, end=end, slots=slots)
            states.move(c.sources, c.slots)
            scores, finished, slots = c.scores, c.finished, c.slots
            history[slots.flatten().long(), k] = c.tokens.flatten()
            if k + 1 < steps:
                logits = self.token(c.tokens.flatten().long(), caches, slots.flatten()).view(B, width, -1)
        return history[slots.long()], scores


def delayed(T, B, delay=3, vocabulary=16, seed=0):
    """Sequences [T + 1, B] whose next token follows from the one `delay` tokens back: the others in between are no help."""
    gen = torch.Generator().manual_seed(seed)
    rows = list(torch.randint(0, vocabulary, (delay, B), generator=gen))
    while len(rows) <= T:
        rows.append((5 * rows[-delay] + 3) % vocabulary)
    return torch.stack(rows[:T + 1])


def main():
    stack = SsmStack()
    for step in range(200):
        s = delayed(64, 32, seed=step).cuda()
        loss = stack.train_step(s[:-1], s[1:])
        if step % 20 == 0:
            print("step %3d  loss %.4f" % (step, float(loss)), flush=True)
    s = delayed(40, 4, seed=1000).cuda()
    caches = stack.caches(4)
    logits = stack.forward(s[:20], caches=caches)[-1]
    right = 0
    for t in range(20, 40):
        token = logits.argmax(-1)
        right += int((token == s[t]).sum())
        logits = stack.token(token, caches)
    print("%d of 80 continued tokens are right" % right)
    found, scores = stack.beams(s[:20], 3, 20)
    print("%d of 80 tokens of the best of three beams are right" % int((found[:, 0].t() == s[20:40]).sum()))
    student = SsmStack(width=32, layers=2, gated=(1,), seed=1)
    for step in range(200):
        s = delayed(64, 32, seed=step).cuda()
        top, index = stack.forward(s[:-1]).topk(4)
        loss = student.distil_step(s[:-1], top, index.int())
        if step % 20 == 0:
            print("step %3d  loss against the first stack %.4f" % (step, float(loss)), flush=True)


if __name__ == "__main__":
    main()
