"""CPU: the oracle of a beam search's step on cases that can be counted by hand, and refusals."""
import ctypes

import numpy as np
import pytest

from oracle import beam
from test_oracle_ssm import EINVAL, EOVERFLOW, EUNSUPPORTED, EWORKSPACE, ONE, Rows, _rows, lib  # noqa: F401

MOST = 0x7FFFFFFF


def test_the_best_of_all_candidates():
    rng = np.random.default_rng(1)
    x, scores = rng.standard_normal((3, 4, 20)), rng.standard_normal((3, 4))
    logp = x - np.log(np.exp(x).sum(-1, keepdims=True))
    flat = (scores[..., None] + logp).reshape(3, 80)
    order = np.argsort(-flat, axis=1, kind="stable")[:, :4]
    new, parents, tokens, done, slots, sources = beam.select(x, scores)
    assert np.array_equal(parents, order // 20) and np.array_equal(tokens, order % 20) and done is slots is sources is None
    assert np.allclose(new, np.take_along_axis(flat, order, 1), rtol=1e-13)


def test_ties_first_steps_and_finished_beams():
    x = np.zeros((1, 3, 5))
    new, parents, tokens, _, _, _ = beam.select(x, np.array([[0.0, -np.inf, -np.inf]]))
    assert parents.tolist() == [[0, 0, 0]] and tokens.tolist() == [[0, 1, 2]] and np.allclose(new, -np.log(5))
    new, parents, tokens, done, _, _ = beam.select(x, np.array([[0.0, -1.0, -9.0]]), np.array([[False, True, False]]), end=4)
    assert parents.tolist() == [[1, 0, 0]] and tokens.tolist() == [[4, 0, 1]] and done.tolist() == [[True, False, False]]
    assert new[0, 0] == -1.0


def test_slots_of_children():
    x = np.zeros((1, 4, 8))
    x[0, 2, 5], x[0, 2, 1], x[0, 1, 7] = 9.0, 8.0, 9.0
    _, parents, _, _, slots, sources = beam.select(x, np.zeros((1, 4)), slots=np.array([[10, 11, 12, 13]]))
    assert parents.tolist() == [[1, 2, 2, 0]]
    assert slots.tolist() == [[11, 12, 13, 10]] and sources.tolist() == [[-1, -1, 12, -1]]


class Beam(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("B", "W", "V", "type", "end")] + [("logits", Rows)] + \
        [(k, ctypes.c_void_p) for k in ("scores", "finished", "slots")]


class Choice(ctypes.Structure):
    _fields_ = [(k, ctypes.c_void_p) for k in ("scores", "parents", "tokens", "finished", "slots", "sources")]


OTHER = 512


def test_bad_arguments_are_rejected_before_any_launch(lib):  # noqa: F811
    size = ctypes.c_size_t

    def call(ws=ONE, n=1 << 40, out=(), **k):
        s, c = Beam(2, 4, 100, 0, -1, _rows(), ONE, None, None), Choice(OTHER, OTHER, OTHER, OTHER, OTHER, OTHER)
        for name, v in k.items():
            setattr(s, name, v)
        for name, v in dict(out).items():
            setattr(c, name, v)
        return lib.bppsa_beam_select(ctypes.byref(s), ctypes.byref(c), ctypes.c_void_p(ws), size(n), None)

    assert lib.bppsa_beam_select(None, None, None, size(0), None) == EINVAL
    for name in ("B", "W", "V"):
        assert call(**{name: 0}) == EINVAL
    assert call(logits=Rows()) == call(scores=None) == EINVAL
    for name in ("scores", "parents", "tokens"):
        assert call(out={name: None}) == EINVAL
    assert call(out={"scores": ONE}) == EINVAL
    assert call(finished=ONE) == call(finished=ONE, end=100) == call(finished=ONE, end=1, out={"finished": None}) == EINVAL
    assert call(finished=OTHER, end=1) == EINVAL
    assert call(slots=ONE, out={"sources": None}) == call(slots=ONE, out={"slots": None}) == call(slots=OTHER) == EINVAL
    assert call(W=33) == call(V=(1 << 19) + 1) == call(type=3) == EUNSUPPORTED
    assert call(B=MOST) == EOVERFLOW
    assert call(ws=None) == call(n=0) == EWORKSPACE
    assert call(ws=ONE + 8) == EINVAL
    f = lib.bppsa_beam_select_workspace_bytes
    f.restype, f.argtypes = size, [ctypes.c_int] * 3
    assert f(MOST, 4, 100) == f(0, 4, 100) == f(1, 33, 100) == f(1, 4, (1 << 19) + 1) == 0
    assert 0 < f(1, 1, 1) < f(64, 8, 1 << 17) < 1 << 24

    one = ctypes.c_void_p(ONE)
    move = lambda t=one, n=4, p=one, rows=2, a=one, b=one, slots=4: lib.bppsa_beam_move(t, ctypes.c_int64(n), p, rows, a, b, slots, None)
    assert move(t=None) == move(n=0) == move(p=None) == move(rows=0) == move(a=None) == move(b=None) == move(slots=0) == EINVAL
    assert move(n=(1 << 22) + 1) == EOVERFLOW


def test_pieces_of_states(lib):  # noqa: F811
    f = lib.bppsa_beam_pieces
    f.restype, f.argtypes = ctypes.c_int64, [ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p]
    n = (ctypes.c_int64 * 3)(1, 16384, 16385)
    pieces = (ctypes.c_int32 * 8)()
    assert f(3, n, None) == f(3, n, pieces) == 4
    assert list(pieces) == [0, 0, 1, 0, 2, 0, 2, 1]
    assert f(1, (ctypes.c_int64 * 1)(0), None) == f(0, n, None) == f(1, None, None) == f(1, (ctypes.c_int64 * 1)(1 << 60), None) == 0


def test_the_binding_refuses_what_is_on_no_gpu(lib):  # noqa: F811
    import torch
    import paper_1907_10134_amd as bp
    with pytest.raises(ValueError):
        bp.beam_select(torch.zeros((2, 4, 10)), torch.zeros((2, 4)))
    with pytest.raises(TypeError):
        bp.beam_select(None, torch.zeros((2, 4)))
    with pytest.raises(ValueError):
        bp.BeamStates([torch.zeros((4, 2))])
    with pytest.raises(TypeError):
        bp.BeamStates([])


def test_the_call_hands_all_its_arguments_over(lib, monkeypatch):  # noqa: F811
    import inspect
    from paper_1907_10134_amd import search
    got = []
    monkeypatch.setattr(search, "_aside", lambda stream, again, *args: got.append((stream, again, args)))
    names = [k for k in inspect.signature(search.beam_select).parameters if k != "stream"]
    search.beam_select(**{k: k for k in names}, stream="side")
    assert got == [("side", search.beam_select, tuple(names))]
