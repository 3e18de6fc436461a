"""fp64 statement of a beam search's step, candidate by candidate.

logits [B, W, V]; scores [B, W]; finished [B, W] bool; slots [B, W].
"""
import numpy as np


def select(logits, scores, finished=None, end=-1, slots=None):
    """(scores, parents, tokens, finished, slots, sources), each [B, W]; the last three None where there are none."""
    B, W, V = logits.shape
    new = np.zeros((B, W))
    parents, tokens = np.zeros((B, W), dtype=int), np.zeros((B, W), dtype=int)
    for b in range(B):
        found = []
        for w in range(W):
            x, score = logits[b, w].astype(np.float64), float(scores[b, w])
            total = np.full(V, -np.inf)
            order = range(V)
            if finished is not None and finished[b, w]:
                if np.isfinite(score):
                    total[end] = score
                    order = [end] + [v for v in range(V) if v != end]
            elif np.isfinite(score):
                with np.errstate(all="ignore"):
                    m = np.max(x)
                    norm = m + np.log(np.sum(np.exp(x - m)))
                if np.isfinite(norm):
                    total = score + (x - norm)
                    order = np.lexsort((np.arange(V), -x))
            found.append([(total[v], w, v) for v in list(order)[:W]])
        for i in range(W):
            best = max((f[0] for f in found if f), key=lambda f: (f[0], -f[1]))
            found[best[1]].pop(0)
            new[b, i], parents[b, i], tokens[b, i] = best
    done = None
    if end >= 0:
        done = tokens == end
        if finished is not None:
            done |= np.take_along_axis(np.asarray(finished), parents, 1)
    if slots is None:
        return new, parents, tokens, done, None, None
    out, sources = np.zeros((B, W), dtype=int), np.full((B, W), -1)
    for b in range(B):
        free = [w for w in range(W) if w not in parents[b]]
        for i, p in enumerate(parents[b]):
            if p in parents[b, :i]:
                out[b, i], sources[b, i] = slots[b, free.pop(0)], slots[b, p]
            else:
                out[b, i] = slots[b, p]
    return new, parents, tokens, done, out, sources
