"""GPU: the loss against a teacher whose numbers are not finite."""
import numpy as np
import pytest

from oracle import distil
from test_gpu_distil import TYPES, _case, _check

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("V", (7, 30, 3000, 40000, 140001))
@pytest.mark.parametrize("dtype,top_type", [(t, t) for t in TYPES] + [("bfloat16", "float32")])
@pytest.mark.parametrize("tail", (False, True))
@pytest.mark.parametrize("hard,temperature", [(0.0, 1.0), (0.4, 2.0)])
def test_a_broken_teacher_breaks_its_own_rows(V, dtype, top_type, tail, hard, temperature):
    """NaN and plus infinity among the entries that count, a NaN for their normaliser: no finite loss and no finite gradient in those
    rows.  Rows beside them, entries that do not count, rows without any and rows of weight zero are as they were."""
    import torch
    import paper_1907_10134_amd as bp
    R = 10
    c, ref = _case(17, R, V, 6, dtype, tail, hard, False, temperature, top_type=top_type)
    weight = torch.ones((R, 1), device="cuda")
    weight[8] = 0.0
    c["weight"], ref["weight"] = weight, weight[:, 0].double().cpu().numpy()

    def put(name, row, k, value):
        c[name][row, 0, k] = value
        ref[name][row, k] = value

    broken = [1, 2, 5]
    put("top_logits", 1, 5, NAN)
    put("top_logits", 2, 0, INF)
    put("top_index", 5, slice(1, None), -1)      # NaN is the row's one entry
    put("top_logits", 5, 0, NAN)
    put("top_logits", 8, 2, NAN)                 # weight zero
    put("top_logits", 9, 4, NAN)                 # these two do not count
    put("top_index", 9, 4, -1)
    put("top_logits", 7, 3, INF)
    put("top_index", 7, 3, V)
    if tail:
        broken.append(0)                         # 4 has no entries and with them no first term
        for row in (0, 4, 8):
            c["top_norm"][row], ref["top_norm"][row] = NAN, NAN
    fine = [k for k in range(R) if k not in broken]
    loss, grad = distil.loss(**ref)
    assert not np.any(np.isfinite(loss[broken])) and not np.any(np.isfinite(grad[broken]))
    got = bp.distil(**c)
    assert not bool(torch.isfinite(got.loss[broken]).any()) and not bool(torch.isfinite(got.dlogits[broken]).any())
    of = lambda d, n: {k: v[fine] if getattr(v, "shape", (0,))[:1] == (n,) else v for k, v in d.items()}
    _check(bp.DistilLoss(got.loss[fine], got.dlogits[fine]), of(c, R), of(ref, R), dtype)
    alone = bp.distil(gradient=False, **c)
    assert torch.equal(alone.loss.nan_to_num(7.0), got.loss.nan_to_num(7.0))


@pytest.mark.parametrize("norm", (-INF, -1000.0))
def test_shares_past_32_bits_break_their_row(norm):
    """A normaliser far below its entries: shares of more than 32 bits hold, no finite loss; without entries it does not matter."""
    import torch
    import paper_1907_10134_amd as bp
    c, ref = _case(18, 5, 50, 6, "float32", True, 0.0, False, 1.0)
    c["top_norm"][2], c["top_norm"][4] = norm, norm          # 4 has no entries
    got = bp.distil(**c)
    assert not bool(torch.isfinite(got.loss[2]).any()) and not bool(torch.isfinite(got.dlogits[2]).any())
    fine = [0, 1, 3, 4]
    _check(bp.DistilLoss(got.loss[fine], got.dlogits[fine]), c, {k: v[fine] if np.ndim(v) else v for k, v in ref.items()}, "float32")
