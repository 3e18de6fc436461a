"""CPU: the fp64 oracle of the gated recurrence against differences, and the library's and the binding's refusals."""
import ctypes

import numpy as np
import pytest

from oracle import gated
from test_oracle_ssm import EINVAL, EOVERFLOW, ESHAPE, EUNSUPPORTED, EWORKSPACE, ONE, Rows, _check_by_differences, _rows, lib  # noqa: F401

MOST = 0x7FFFFFFF


def _layer(rng, T, B, D, gate, given):
    x = {k: rng.standard_normal((T, B, D)) for k in ("x", "r", "i") + (("z",) if gate else ())}
    x["decay"] = rng.uniform(0.2, 2.0, D)
    if given:
        x.update(r_bias=rng.standard_normal(D), i_bias=rng.standard_normal(D), h0=rng.standard_normal((B, D)))
    return x


@pytest.mark.parametrize("gate,given,lengths", [(False, False, None), (True, True, None), (True, True, (5, 0, 1))])
def test_gradients_against_differences(gate, given, lengths):
    rng = np.random.default_rng(3)
    x = _layer(rng, 7, 3, 4, gate, given)
    dy, dh_last = rng.standard_normal((7, 3, 4)), rng.standard_normal((3, 4))

    def f():
        y, last, _ = gated.scan(**x, lengths=lengths)
        return float((y * dy).sum() + (last * dh_last).sum())

    _check_by_differences(f, x, gated.scan_backward(dy, **x, lengths=lengths, dh_last=dh_last), rng)


def test_a_sequence_in_two_parts_is_the_whole():
    rng = np.random.default_rng(5)
    x = _layer(rng, 9, 2, 4, True, True)
    whole, last, _ = gated.scan(**x)
    cut = lambda a, b: {k: v[a:b] if k in ("x", "r", "i", "z") else v for k, v in x.items()}
    y1, h1, _ = gated.scan(**cut(0, 4))
    y2, h2, _ = gated.scan(**dict(cut(4, 9), h0=h1))
    assert np.allclose(np.concatenate((y1, y2)), whole, rtol=1e-13) and np.allclose(h2, last, rtol=1e-13)


class Layer(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("T", "B", "D", "type")] + [(k, Rows) for k in ("x", "r", "i", "z")] + \
        [(k, ctypes.c_void_p) for k in ("decay", "r_bias", "i_bias", "h0", "lengths")]


class Grads(ctypes.Structure):
    _fields_ = [(k, Rows) for k in ("dx", "dr", "di", "dz")] + [(k, ctypes.c_void_p) for k in ("ddecay", "dr_bias", "di_bias", "dh0")]


def _gated(**k):
    l = Layer(16, 2, 64, 0, _rows(), _rows(), _rows(), Rows(), ONE, None, None, None, None)
    for name, v in k.items():
        setattr(l, name, v)
    return l


def _bytes(lib, name):  # noqa: F811
    f = getattr(lib, "bppsa_gated_" + name)
    f.restype, f.argtypes = ctypes.c_size_t, [ctypes.c_int] * 3
    return f


def test_byte_counts(lib):  # noqa: F811
    for name in ("scan_states_bytes", "scan_backward_workspace_bytes"):
        f = _bytes(lib, name)
        assert 0 < f(1, 1, 1) <= f(1000, 16, 640) < 1 << 30
        assert f(0, 1, 1) == f(MOST, MOST, MOST) == f(1, 1, (1 << 24) + 1) == 0
        assert f(64, 1 << 17, 64 * 64) == 0            # 2^23 tiles
    assert _bytes(lib, "scan_workspace_bytes")(MOST, MOST, MOST) == 0


def test_bad_arguments_are_rejected_before_any_launch(lib):  # noqa: F811
    size, y, big = ctypes.c_size_t, ctypes.byref(_rows()), 1 << 40
    scan = lambda l, out=y, last=None, states=None, ws=ONE, n=big: lib.bppsa_gated_scan(
        None if l is None else ctypes.byref(l), out, last, states, ctypes.c_void_p(ws), size(n), None)
    assert scan(None) == EINVAL
    for name in ("T", "B", "D"):
        assert scan(_gated(**{name: 0})) == EINVAL
    assert scan(_gated(x=Rows())) == scan(_gated(r=Rows())) == scan(_gated(i=Rows())) == scan(_gated(decay=None)) == EINVAL
    assert scan(_gated(type=3)) == scan(_gated(type=-1)) == EUNSUPPORTED
    assert scan(_gated(D=1 << 25)) == scan(_gated(T=MOST)) == scan(_gated(T=1 << 20, B=1 << 16)) == EOVERFLOW
    assert scan(_gated(), out=None) == scan(_gated(), out=ctypes.byref(Rows(ONE, 0, 64))) == EINVAL
    assert scan(_gated(h0=ONE), last=ctypes.c_void_p(ONE)) == scan(_gated(), states=ctypes.c_void_p(ONE + 4)) == EINVAL

    def back(l, dy=y, states=ONE, last=None, ws=ONE, n=big, **k):
        g = Grads(_rows(), _rows(), _rows(), Rows(), ONE, None, None, None)
        for name, v in k.items():
            setattr(g, name, v)
        return lib.bppsa_gated_scan_backward(ctypes.byref(l), dy, last, ctypes.c_void_p(states), ctypes.byref(g), ctypes.c_void_p(ws),
                                             size(n), None)

    assert back(_gated(), states=None) == back(_gated(), states=ONE + 8) == back(_gated(), dy=None) == EINVAL
    assert back(_gated(), ddecay=None) == back(_gated(), dx=Rows()) == back(_gated(), dr=Rows()) == back(_gated(), di=Rows()) == EINVAL
    assert back(_gated(), dz=_rows()) == back(_gated(z=_rows())) == EINVAL           # one without the other
    assert back(_gated(), dx=Rows(ONE, 64, 0)) == EINVAL
    assert back(_gated(), last=ctypes.c_void_p(ONE), dh0=ONE) == EINVAL
    assert back(_gated(), n=0) == back(_gated(), ws=None) == EWORKSPACE
    assert back(_gated(), ws=ONE + 16) == EINVAL
    step = lambda l, state=ONE, n=4, slots=None: lib.bppsa_gated_scan_step(ctypes.byref(l), y, ctypes.c_void_p(state), n, slots, None)
    assert step(_gated()) == ESHAPE and step(_gated(T=1, B=5)) == ESHAPE
    assert step(_gated(T=1), state=None) == step(_gated(T=1), n=0) == step(_gated(T=1, h0=ONE)) == step(_gated(T=1, lengths=ONE)) == EINVAL


def test_the_binding_refuses_what_is_on_no_gpu(lib):  # noqa: F811
    import torch
    import paper_1907_10134_amd as bp
    x, decay = torch.zeros((4, 2, 8)), torch.ones(8)
    with pytest.raises(ValueError):
        bp.gated_scan(x, x, x, decay)
    with pytest.raises(ValueError):
        bp.gated_scan_step(x[0], x[0], x[0], decay, torch.zeros((2, 8)))
    with pytest.raises(TypeError):
        bp.gated_scan(None, x, x, decay)
    with pytest.raises(ValueError):
        bp.gated_scan(x[0], x, x, decay)
    with pytest.raises(ValueError):
        bp.gated_scan_states(0, 1, 1)


@pytest.mark.parametrize("name", ("gated_scan", "gated_scan_backward", "gated_scan_step"))
def test_every_call_hands_all_its_arguments_over(lib, monkeypatch, name):  # noqa: F811
    import inspect
    from paper_1907_10134_amd import gated as module
    call, got = getattr(module, name), []
    monkeypatch.setattr(module, "_aside", lambda stream, again, *args: got.append((stream, again, args)))
    names = [k for k in inspect.signature(call).parameters if k != "stream"]
    assert list(inspect.signature(call).parameters)[-1] == "stream"
    call(**{k: k for k in names}, stream="side")
    assert got == [("side", call, tuple(names))]
