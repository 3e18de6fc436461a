"""A small stack of selective state space layers, trained and served with the library's operators.

A layer: root-mean-square norm, a projection to two halves, the short convolution and the selective scan of the first half
gated by the second, a projection back that is added to the stream.  The projections, norms and the loss are plain torch;
the convolution, the scan, their gradients, their single-token steps and the optimiser are the library's.  Activations are
bfloat16, the stream between the layers and all parameters float32; the projections use the bfloat16 copies that the
optimiser keeps.

    python -m workloads.ssm_stack        trains on sequences with a delayed rule and continues some token by token
"""
from __future__ import annotations

import math

import torch

import paper_1907_10134_amd as bp

BF16 = torch.bfloat16
DECAYED = ("embed", "in_proj", "x_proj", "dt_proj", "out_proj")


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
    def __init__(self, vocabulary=16, width=64, layers=2, states=16, taps=4, state_bits=8, lr=3e-3, seed=0, device="cuda"):
        gen = torch.Generator().manual_seed(seed)
        normal = lambda scale, *shape: torch.randn(shape, generator=gen) * scale
        uniform = lambda lo, hi, *shape: lo + (hi - lo) * torch.rand(shape, generator=gen)
        d, D, N, R = width, 2 * width, states, -(-width // 16)
        self.sizes, self.layers, self.taps = (d, D, N, R), layers, taps
        p = {"embed": normal(0.3, vocabulary, d), "last_norm": torch.ones(d)}
        for l in range(layers):
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
        states [B, D, N], last inputs [B, taps - 1, D]) of each layer, filled with the state after each sample."""
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
        p, w, g, keep = self.p, self.w, self.g, []
        D = self.sizes[1]
        T, B = tokens.shape
        logits = self.forward(tokens, lengths, keep)
        logp = torch.log_softmax(logits, -1)
        real = torch.ones((T, B), device=logits.device) if lengths is None else \
            (torch.arange(T, device=logits.device)[:, None] < lengths).float()
        real = real / real.sum()
        loss = -(logp.gather(-1, targets[..., None])[..., 0] * real).sum()
        dlogits = torch.exp(logp)
        dlogits.scatter_add_(-1, targets[..., None], torch.full((T, B, 1), -1.0, device=logits.device))
        dlogits = (dlogits * real[..., None]).to(BF16)
        outer = lambda a, b: torch.mm(a.flatten(0, -2).t(), b.flatten(0, -2)).float()        # sum over tokens of a b^T
        back = lambda a, weight: torch.mm(a.flatten(0, -2), weight).unflatten(0, a.shape[:-1])
        x, r, n = keep.pop()
        dembed = outer(dlogits, n)
        dx, dw = _norm_backward(back(dlogits, w["embed"]).float(), x, r, p["last_norm"])
        g["last_norm"].copy_(dw)
        for l in reversed(range(self.layers)):
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
            k = bp.ssm_conv_backward(dc, u, p["conv_w%d" % l], p["conv_b%d" % l], lengths=lengths)
            g["conv_w%d" % l].copy_(k.dweight)
            g["conv_b%d" % l].copy_(k.dbias)
            dxz = torch.cat((k.dx, s.dz), -1)
            g["in_proj%d" % l].copy_(outer(dxz, n))
            dn, dw = _norm_backward(back(dxz, w["in_proj%d" % l]).float(), x, r, p["norm%d" % l])
            g["norm%d" % l].copy_(dw)
            dx = dx + dn
        g["embed"].copy_(dembed.index_add_(0, tokens.flatten(), dx.flatten(0, 1)))
        self.optimiser.step()
        return loss

    def caches(self, slots, device="cuda"):
        """Empty states of `slots` streams: (scan [slots, D, N] float32, convolution [slots, taps - 1, D]) of each layer."""
        _, D, N, _ = self.sizes
        return [(torch.zeros((slots, D, N), device=device), torch.zeros((slots, self.taps - 1, D), dtype=BF16, device=device))
                for _ in range(self.layers)]

    def token(self, tokens, caches, slots=None):
        """Logits [B, vocabulary] behind one more token [B] of the streams in `slots`, whose states move on."""
        p, w = self.p, self.w
        D = self.sizes[1]
        x = p["embed"][tokens]
        for l in range(self.layers):
            h, last = caches[l]
            xz = _mm(_norm(x, p["norm%d" % l])[0].to(BF16), w["in_proj%d" % l])
            c = bp.ssm_conv_step(xz[:, :D], p["conv_w%d" % l], p["conv_b%d" % l], last, slots=slots)
            low, Bm, Cm = self._cut(_mm(c, w["x_proj%d" % l]))
            y = bp.ssm_scan_step(c, _mm(low, w["dt_proj%d" % l]), -torch.exp(p["A_log%d" % l]), Bm, Cm, h,
                                 skip=p["skip%d" % l], z=xz[:, D:], dt_bias=p["dt_bias%d" % l], slots=slots)
            x = x + _mm(y, w["out_proj%d" % l]).float()
        return _mm(_norm(x, p["last_norm"])[0].to(BF16), w["embed"]).float()


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


if __name__ == "__main__":
    main()
