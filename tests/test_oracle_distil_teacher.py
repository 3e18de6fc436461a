"""CPU: the fp64 oracle of the loss against a teacher whose numbers are not finite, against the formula in torch."""
import numpy as np
import pytest

from oracle import distil

NAN, INF = float("nan"), float("inf")


def _formula(x, top, index, norm):
    """The loss and its gradient of one row at temperature 1, by differentiating what the header says."""
    import torch
    x = torch.tensor(x, dtype=torch.float64, requires_grad=True)
    on = [k for k in range(len(index)) if 0 <= index[k] < len(x) and not top[k] == -INF]
    c, t = torch.tensor([index[k] for k in on], dtype=torch.long), torch.tensor([top[k] for k in on], dtype=torch.float64)
    logq = torch.log_softmax(x, 0)
    logp = torch.log_softmax(t, 0) if norm is None else t - norm
    p = torch.exp(logp)
    loss = (p * (logp - logq[c])).sum()
    if norm is not None:
        p0 = 1 - p.sum()
        others = torch.ones(len(x), dtype=torch.bool)
        others[c] = False
        loss = loss + p0 * (torch.log(p0) - torch.log(torch.exp(logq)[others].sum()))
    return float(loss.detach()), torch.autograd.grad(loss, x)[0].numpy()


@pytest.mark.parametrize("top,index,norm", [([NAN, 1.0, 0.5], [0, 2, 4], None), ([INF, 1.0, 0.5], [0, 2, 4], None),
                                            ([NAN, 1.0, 0.5], [0, 2, 4], 2.5), ([1.0, 0.5, 0.0], [0, 2, 4], NAN),
                                            ([NAN, 1.0, 0.5], [0, -1, -1], None)])
def test_a_broken_teacher_breaks_its_row(top, index, norm):
    x = np.random.default_rng(1).standard_normal((1, 7))
    loss, grad = distil.loss(x, np.array([top]), np.array([index]), top_norm=None if norm is None else np.array([norm]))
    want, want_grad = _formula(x[0], top, index, norm)
    assert np.isnan(want) and np.isnan(loss[0]) and np.all(np.isnan(want_grad)) and np.all(np.isnan(grad))


def test_a_row_without_entries_has_no_first_term_whatever_its_normaliser():
    x = np.random.default_rng(2).standard_normal((1, 7))
    loss, grad = distil.loss(x, np.zeros((1, 2)), np.full((1, 2), -1), top_norm=np.array([NAN]))
    assert abs(loss[0]) < 1e-15 and np.max(np.abs(grad)) < 1e-15


@pytest.mark.parametrize("norm", [None, 2.5])
def test_what_does_not_count_may_be_anything(norm):
    x = np.random.default_rng(3).standard_normal((1, 7))
    more = dict(top_norm=None if norm is None else np.array([norm]))
    want = distil.loss(x, np.array([[1.0, 0.5]]), np.array([[3, 5]]), **more)
    got = distil.loss(x, np.array([[NAN, 1.0, INF, 0.5]]), np.array([[-1, 3, 7, 5]]), **more)
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1]) and np.all(np.isfinite(got[1]))
