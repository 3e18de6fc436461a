"""GPU: the loss with the others as one more class, of a student to whom those others are next to impossible."""
import numpy as np
import pytest

from test_gpu_distil import TYPES, _check, _on

pytestmark = pytest.mark.gpu


def _case(V, dtype, temperature, hard, far, weights):
    """Eight entries at one largest logit, some other tokens `far` below it, all else masked; the teacher gives the others one half."""
    import torch
    R = len(far)
    rng = np.random.default_rng(V)
    x = np.full((R, V), -np.inf)
    index = np.zeros((R, 8), dtype=np.int32)
    targets = np.full(R, -1)
    for k, distances in enumerate(far):
        places = rng.permutation(V)[:8 + len(distances)]
        index[k] = places[:8]
        x[k, places[:8]] = 1.5
        x[k, places[8:]] = 1.5 - temperature * np.array(distances)
        if hard and k % 3:                     # an entry, one of the others, none
            targets[k] = places[0 if k % 3 == 1 or not len(distances) else 8]
    t = getattr(torch, dtype)
    c = {"logits": _on(x, t).view(R, 1, V), "top_logits": torch.full((R, 1, 8), float(np.log(0.5 / 8)) * temperature, device="cuda"),
         "top_index": _on(index, torch.int32).view(R, 1, 8), "top_norm": torch.zeros((R, 1), device="cuda"),
         "weight": torch.tensor(weights, device="cuda").view(R, 1)}
    if hard:
        c["targets"] = _on(targets, torch.int32).view(R, 1)
    ref = {k: v.double().cpu().numpy()[:, 0] for k, v in c.items()}
    ref["top_index"] = index.astype(int)
    if hard:
        ref["targets"] = targets
    more = dict(temperature=temperature, hard=hard)
    return dict(c, **more), dict(ref, **more)


FAR = ([86.5], [80.0], [86.0, 84.5, 80.5], [45.0, 44.5, 86.0], [44.0, 60.0], [2.0, 80.0], [])
WEIGHTS = {"float16": (1.0, 2.0 ** 14, 2.0 ** 14, 2.0 ** -10, 2.0 ** 14, 2.0 ** 14, 1.0),
           "bfloat16": (1.0, 65536.0, 65536.0, 2.0 ** -10, 2.0 ** 40, 65536.0, 1.0)}
WEIGHTS["float32"] = WEIGHTS["bfloat16"]


@pytest.mark.parametrize("V", (40, 3000, 40000, 140001))
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("temperature,hard", [(1.0, 0.0), (1.0, 0.3), (2.0, 0.4), (0.5, 1.0)])
def test_others_that_are_next_to_impossible(V, dtype, temperature, hard):
    """Shares of the others from 2^-63 to 2^-125 of the largest, under weights as large as a scaled loss has: their gradient is the
    weight times the teacher's half, dealt out among them, and zero at tokens that are masked.  An exponential's argument of up to 125
    in base two is rounded to 2^-18, which is 45 of 2^-24 in a share of the half: less than the 64 and more that are let by."""
    import torch
    import paper_1907_10134_amd as bp
    c, ref = _case(V, dtype, temperature, hard, FAR, WEIGHTS[dtype])
    got = bp.distil(**c)
    masked = torch.isinf(c["logits"])
    assert bool((got.dlogits[masked] == 0).all())
    _check(got, c, ref, dtype)
    place = bp.distil(dlogits=c["logits"], **c)
    assert torch.equal(place.dlogits, got.dlogits) and torch.equal(place.loss, got.loss)
