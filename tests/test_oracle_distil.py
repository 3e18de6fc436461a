"""CPU: the fp64 oracle of the loss against a teacher's top logits against differences and torch, and refusals."""
import ctypes

import numpy as np
import pytest

from oracle import distil
from test_oracle_ssm import EINVAL, EOVERFLOW, EUNSUPPORTED, ONE, Rows, _rows, lib  # noqa: F401

MOST = 0x7FFFFFFF


def _case(rng, R=4, V=11, K=5):
    index = np.stack([rng.permutation(V)[:K] for _ in range(R)])
    index[1, 3:] = -1
    index[2] = -1
    return dict(logits=rng.standard_normal((R, V)), top_logits=2 * rng.standard_normal((R, K)), top_index=index)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("temperature,hard", [(1.0, 0.0), (2.0, 0.3), (0.5, 1.0)])
def test_gradient_against_differences(tail, temperature, hard):
    rng = np.random.default_rng(1)
    x = _case(rng)
    more = dict(temperature=temperature, hard=hard, targets=np.array([3, -1, 2, 10]), weight=np.array([1.0, 2.0, 0.0, 0.5]))
    if tail:
        more["top_norm"] = np.log(np.exp(x["top_logits"] / temperature).sum(1) + 0.7)
    _, grad = distil.loss(**x, **more)
    for at in [(0, 0), (0, 3), (1, 5), (3, 10), (3, 1), (2, 2)] + [(0, int(x["top_index"][0, 0])), (3, int(x["top_index"][3, 4]))]:
        up, down = (dict(x, logits=x["logits"].copy()) for _ in range(2))
        up["logits"][at] += 1e-5
        down["logits"][at] -= 1e-5
        got = (distil.loss(**up, **more)[0].sum() - distil.loss(**down, **more)[0].sum()) / 2e-5
        assert abs(got - grad[at]) <= 1e-8, at


def test_all_tokens_as_entries_are_the_divergence_of_two_softmaxes():
    import torch
    rng = np.random.default_rng(2)
    x = _case(rng, V=5, K=5)
    x["top_index"][:] = np.arange(5)
    student, teacher = torch.from_numpy(x["logits"]), torch.from_numpy(x["top_logits"])
    want = torch.nn.functional.kl_div(torch.log_softmax(student, 1), torch.softmax(teacher, 1), reduction="none").sum(1)
    assert np.allclose(distil.loss(**x)[0], want.numpy(), rtol=1e-12)


class Distil(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("T", "B", "V", "K", "type", "top_type")] + [("logits", Rows)] + \
        [(k, ctypes.c_void_p) for k in ("top_logits", "top_index", "top_norm", "weight", "targets")] + \
        [("temperature", ctypes.c_float), ("hard", ctypes.c_float)]


def test_bad_arguments_are_rejected_before_any_launch(lib):  # noqa: F811
    def call(loss=ONE, dlogits=None, **k):
        r = Distil(4, 2, 16, 4, 0, 0, _rows(), ONE, ONE, None, None, None, 1.0, 0.0)
        for name, v in k.items():
            setattr(r, name, v)
        return lib.bppsa_distil(ctypes.byref(r), ctypes.c_void_p(loss), dlogits, None)

    assert lib.bppsa_distil(None, ctypes.c_void_p(ONE), None, None) == EINVAL
    for name in ("T", "B", "V", "K"):
        assert call(**{name: 0}) == EINVAL
    assert call(logits=Rows()) == call(top_logits=None) == call(top_index=None) == call(loss=None) == EINVAL
    for bad in (0.0, -1.0, float("inf"), float("nan")):
        assert call(temperature=bad) == EINVAL
    assert call(hard=-0.1) == call(hard=1.1) == call(hard=float("nan")) == call(hard=0.5) == EINVAL       # the last: no targets
    assert call(dlogits=ctypes.byref(Rows(ONE, 0, 64))) == EINVAL
    assert call(dlogits=ctypes.byref(Rows(ONE, 128, 64))) == EINVAL                # the logits' memory in another order
    assert call(K=257) == call(type=3) == call(top_type=-1) == EUNSUPPORTED
    assert call(T=MOST, B=MOST) == call(V=(1 << 20) + 1) == call(T=1 << 22, B=1, V=1) == EOVERFLOW


def test_the_binding_refuses_what_is_on_no_gpu(lib):  # noqa: F811
    import torch
    import paper_1907_10134_amd as bp
    x, top, index = torch.zeros((4, 16)), torch.zeros((4, 3)), torch.zeros((4, 3), dtype=torch.int32)
    with pytest.raises(ValueError):
        bp.distil(x, top, index)
    with pytest.raises(TypeError):
        bp.distil(None, top, index)
    with pytest.raises(ValueError):
        bp.distil(x, top, index, hard=0.5)
    with pytest.raises(ValueError):
        bp.distil(x, top[:3], index)


def test_the_call_hands_all_its_arguments_over(lib, monkeypatch):  # noqa: F811
    import inspect
    from paper_1907_10134_amd import distil as call
    module = inspect.getmodule(call)
    got = []
    monkeypatch.setattr(module, "_aside", lambda stream, again, *args: got.append((stream, again, args)))
    names = [k for k in inspect.signature(call).parameters if k != "stream"]
    assert list(inspect.signature(call).parameters)[-1] == "stream"
    call(**{k: k for k in names}, stream="side")
    assert got == [("side", call, tuple(names))]
