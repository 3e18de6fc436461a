"""CPU: the fp64 state space oracle against differences, and the binding's and the library's refusals."""
import ctypes
import os

import numpy as np
import pytest

from oracle import ssm

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _layer(rng, T, B, D, N, G, gate, given):
    x = dict(u=rng.standard_normal((T, B, D)), dt=rng.standard_normal((T, B, D)), A=-rng.uniform(0.2, 3.0, (D, N)),
             Bm=rng.standard_normal((T, B, G, N)), Cm=rng.standard_normal((T, B, G, N)))
    if gate:
        x["z"] = rng.standard_normal((T, B, D))
    if given:
        x.update(skip=rng.standard_normal(D), dt_bias=rng.standard_normal(D), h0=rng.standard_normal((B, D, N)))
    return x


# a central difference of step e is off by about e^2 f''' / 6 and 2^-53 f / e: 1e-10 and 1e-10 of values of order one at 1e-6
# to 1e-5, of sums of some tens of terms 1e-8
EPS, TOL = 1e-5, 1e-7


def _check_by_differences(f, inputs, grads, rng, tries=6):
    for name, x in inputs.items():
        g = grads["d" + name]
        for _ in range(tries):
            at = tuple(rng.integers(0, k) for k in x.shape)
            was = x[at]
            x[at] = was + EPS
            up = f()
            x[at] = was - EPS
            down = f()
            x[at] = was
            assert abs((up - down) / (2 * EPS) - g[at]) <= TOL * max(1.0, abs(g[at])), (name, at)


@pytest.mark.parametrize("gate,given,lengths", [(False, False, None), (True, True, None), (True, True, (5, 0, 1))])
def test_scan_gradients_against_differences(gate, given, lengths):
    rng = np.random.default_rng(3)
    x = _layer(rng, 7, 3, 4, 3, 2, gate, given)
    dy = rng.standard_normal((7, 3, 4))
    f = lambda: float((ssm.scan(**x, lengths=lengths)[0] * dy).sum())
    _check_by_differences(f, x, ssm.scan_backward(dy, **x, lengths=lengths), rng)


@pytest.mark.parametrize("silu", [False, True])
@pytest.mark.parametrize("lengths", [None, (6, 0, 1)])
def test_conv_gradients_against_differences(silu, lengths):
    rng = np.random.default_rng(4)
    x = dict(x=rng.standard_normal((6, 3, 5)), weight=rng.standard_normal((5, 4)), bias=rng.standard_normal(5),
             state0=rng.standard_normal((3, 3, 5)))
    dy = rng.standard_normal((6, 3, 5))
    f = lambda: float((ssm.conv(**x, silu=silu, lengths=lengths)[0] * dy).sum())
    _check_by_differences(f, x, ssm.conv_backward(dy, **x, silu=silu, lengths=lengths), rng)


def test_a_sequence_in_two_parts_is_the_whole():
    rng = np.random.default_rng(5)
    x = _layer(rng, 9, 2, 4, 3, 1, True, True)
    whole, last, _, _ = ssm.scan(**x)
    cut = lambda a, b: {k: v[a:b] if k in ("u", "dt", "z", "Bm", "Cm") else v for k, v in x.items()}
    y1, h1, _, _ = ssm.scan(**cut(0, 4))
    y2, h2, _, _ = ssm.scan(**dict(cut(4, 9), h0=h1))
    assert np.allclose(np.concatenate((y1, y2)), whole, rtol=1e-13) and np.allclose(h2, last, rtol=1e-13)


def test_e4m3_values_are_torchs():
    import torch
    all_ = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(all_, ssm.e4m3_values())


# ---- refusals -------------------------------------------------------------------------------------

class Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("st", ctypes.c_int64), ("sb", ctypes.c_int64)]


class Layer(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("T", "B", "D", "N", "G", "type")] + \
        [(k, Rows) for k in ("u", "dt", "z", "Bm", "Cm")] + [(k, ctypes.c_void_p) for k in ("A", "skip", "dt_bias", "h0", "lengths")]


class Grads(ctypes.Structure):
    _fields_ = [(k, Rows) for k in ("du", "ddt", "dz")] + \
        [(k, ctypes.c_void_p) for k in ("dBm", "dCm", "dA", "dskip", "ddt_bias", "dh0")]


class Conv(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("T", "B", "D", "W", "type", "silu")] + [("x", Rows)] + \
        [(k, ctypes.c_void_p) for k in ("weight", "bias", "state0", "lengths")]


ONE = 256                     # a non-null pointer that is never dereferenced
EINVAL, ESHAPE, EWORKSPACE, EOVERFLOW, EUNSUPPORTED = 1, 2, 3, 4, 6


@pytest.fixture(scope="module")
def lib():
    path = os.path.join(ROOT, "paper_1907_10134_amd", "libbppsa.so")
    if not os.path.exists(path):
        import __graft_entry__
        __graft_entry__.build()
    lib = ctypes.CDLL(path)
    for name, args in (("scan_states_bytes", 4), ("scan_workspace_bytes", 5), ("scan_backward_workspace_bytes", 5),
                       ("conv_backward_workspace_bytes", 4)):
        f = getattr(lib, "bppsa_ssm_" + name)
        f.restype, f.argtypes = ctypes.c_size_t, [ctypes.c_int] * args
    return lib


def _rows():
    return Rows(ONE, 64, 64)


def _ssm(T=8, B=2, D=32, N=16, G=1, type=0, **other):
    l = Layer(T, B, D, N, G, type, _rows(), _rows(), Rows(), _rows(), _rows(), ONE, None, None, None, None)
    for k, v in other.items():
        setattr(l, k, v)
    return l


def _call_scan(lib, l, y=_rows(), ws=0, nbytes=0):
    return lib.bppsa_ssm_scan(ctypes.byref(l) if l else None, ctypes.byref(y) if y else None, None, None, ctypes.c_void_p(ws),
                              ctypes.c_size_t(nbytes), None)


def test_scan_refusals(lib):
    assert _call_scan(lib, None) == EINVAL and _call_scan(lib, _ssm(), y=None) == EINVAL
    assert _call_scan(lib, _ssm(), y=Rows()) == EINVAL
    for bad in (dict(T=0), dict(B=0), dict(D=-1), dict(N=0), dict(G=0), dict(u=Rows()), dict(Cm=Rows()), dict(A=None)):
        assert _call_scan(lib, _ssm(**bad)) == EINVAL, bad
    assert _call_scan(lib, _ssm(G=3)) == ESHAPE
    assert _call_scan(lib, _ssm(N=65)) == EUNSUPPORTED and _call_scan(lib, _ssm(type=3)) == EUNSUPPORTED
    assert _call_scan(lib, _ssm(T=1 << 30, B=1 << 15, D=1 << 20)) == EOVERFLOW
    # outputs of which two elements share a place
    assert _call_scan(lib, _ssm(), y=Rows(ONE, 0, 64)) == EINVAL and _call_scan(lib, _ssm(), y=Rows(ONE, 64, 0)) == EINVAL
    # the last states in the place of the first ones
    assert lib.bppsa_ssm_scan(ctypes.byref(_ssm(h0=ONE)), ctypes.byref(_rows()), ctypes.c_void_p(ONE), None, ctypes.c_void_p(512),
                              ctypes.c_size_t(1 << 40), None) == EINVAL
    need = lib.bppsa_ssm_scan_workspace_bytes(4000, 1, 32, 16, 1)
    if need:
        assert _call_scan(lib, _ssm(T=4000, B=1)) == EWORKSPACE
        assert _call_scan(lib, _ssm(T=4000, B=1), ws=512, nbytes=need - 1) == EWORKSPACE
        assert _call_scan(lib, _ssm(T=4000, B=1), ws=260, nbytes=need) == EINVAL


def test_scan_backward_refusals(lib):
    def call(l, states=ONE, dy=_rows(), ws=512, nbytes=1 << 40, **other):
        g = Grads(_rows(), _rows(), Rows(), ONE, ONE, ONE, None, None, None)
        for k, v in other.items():
            setattr(g, k, v)
        return lib.bppsa_ssm_scan_backward(ctypes.byref(l), ctypes.byref(dy), ctypes.c_void_p(states), ctypes.byref(g),
                                           ctypes.c_void_p(ws), ctypes.c_size_t(nbytes), None)

    assert call(_ssm(), states=None) == EINVAL and call(_ssm(), dy=Rows()) == EINVAL
    assert call(_ssm(), dA=None) == EINVAL and call(_ssm(), dBm=None) == EINVAL and call(_ssm(), du=Rows()) == EINVAL
    assert call(_ssm(z=_rows())) == EINVAL and call(_ssm(), dz=_rows()) == EINVAL      # a gate without its gradient, and the reverse
    assert call(_ssm(), ddt=Rows(ONE, 0, 64)) == EINVAL
    assert call(_ssm(), ws=None) == EWORKSPACE and call(_ssm(), ws=260) == EINVAL
    assert call(_ssm(), nbytes=lib.bppsa_ssm_scan_backward_workspace_bytes(8, 2, 32, 16, 1) - 1) == EWORKSPACE
    assert call(_ssm(G=5)) == ESHAPE and call(_ssm(N=100)) == EUNSUPPORTED


def test_step_and_conv_refusals(lib):
    def step(l, state=ONE, slots=4):
        return lib.bppsa_ssm_scan_step(ctypes.byref(l), ctypes.byref(_rows()), ctypes.c_void_p(state), slots, None, None)

    assert step(_ssm(T=2)) == ESHAPE and step(_ssm(T=1), state=None) == EINVAL and step(_ssm(T=1), slots=0) == EINVAL
    assert step(_ssm(T=1, h0=ONE)) == EINVAL and step(_ssm(T=1, lengths=ONE)) == EINVAL
    assert step(_ssm(T=1, B=5)) == ESHAPE                # more rows than slots, and no list of slots

    def conv(T=8, B=2, D=32, W=4, type=0, y=_rows(), **other):
        c = Conv(T, B, D, W, type, 1, _rows(), ONE, None, None, None)
        for k, v in other.items():
            setattr(c, k, v)
        return c, lib.bppsa_ssm_conv(ctypes.byref(c), ctypes.byref(y), None, None)

    assert conv(T=0)[1] == EINVAL and conv(x=Rows())[1] == EINVAL and conv(weight=None)[1] == EINVAL
    assert conv(W=1)[1] == EUNSUPPORTED and conv(W=5)[1] == EUNSUPPORTED and conv(type=-1)[1] == EUNSUPPORTED
    assert conv(y=Rows(ONE, 0, 64))[1] == EINVAL and conv(B=1 << 17)[1] == EOVERFLOW
    c = Conv(8, 2, 32, 4, 0, 1, _rows(), ONE, None, None, None)
    back = lambda c, dx=_rows(), dw=ONE, ws=512, nbytes=1 << 40: lib.bppsa_ssm_conv_backward(
        ctypes.byref(c), ctypes.byref(_rows()), ctypes.byref(dx), ctypes.c_void_p(dw), None, None, ctypes.c_void_p(ws),
        ctypes.c_size_t(nbytes), None)
    assert back(c, dx=Rows()) == EINVAL and back(c, dw=None) == EINVAL and back(c, ws=None) == EWORKSPACE
    assert back(c, nbytes=lib.bppsa_ssm_conv_backward_workspace_bytes(8, 2, 32, 4) - 1) == EWORKSPACE
    c.T = 2
    assert lib.bppsa_ssm_conv_step(ctypes.byref(c), ctypes.byref(_rows()), ctypes.c_void_p(ONE), 4, None, None) == ESHAPE


def test_sizes_queries(lib):
    assert lib.bppsa_ssm_scan_states_bytes(0, 1, 1, 1) == 0 and lib.bppsa_ssm_scan_states_bytes(1, 1, 1, 65) == 0
    assert lib.bppsa_ssm_scan_states_bytes(17, 3, 5, 7) >= 3 * 3 * 5 * 7 * 4 // 3
    assert lib.bppsa_ssm_scan_backward_workspace_bytes(8, 2, 30, 16, 4) == 0          # D is no multiple of G
    assert lib.bppsa_ssm_conv_backward_workspace_bytes(8, 2, 30, 1) == 0
    # sizes past 32 bits
    assert lib.bppsa_ssm_scan_states_bytes(1 << 20, 64, 8192, 16) > 1 << 32


def test_adamw_pieces(lib):
    lib.bppsa_adamw_pieces.restype = ctypes.c_int64
    n = (ctypes.c_int64 * 4)(1, 4096, 0, 4097)
    assert lib.bppsa_adamw_pieces(4, n, None) == 4
    out = (ctypes.c_int32 * 8)()
    assert lib.bppsa_adamw_pieces(4, n, out) == 4 and list(out) == [0, 0, 1, 0, 3, 0, 3, 1]
    assert lib.bppsa_adamw_pieces(0, n, None) == 0 and lib.bppsa_adamw_pieces(1, (ctypes.c_int64 * 1)(-1), None) == 0
    one, d = ctypes.c_void_p(ONE), ctypes.c_double
    call = lambda nt=1, np_=1, bits=32, step=1, b1=0.9, gt=0, eps=1e-8, t=one: lib.bppsa_adamw_step(
        nt, t, ctypes.c_int64(np_), one, gt, bits, step, d(1e-3), d(b1), d(0.999), d(eps), ctypes.c_uint32(0), None)
    assert call(nt=0) == EINVAL and call(np_=0) == EINVAL and call(step=0) == EINVAL and call(b1=1.0) == EINVAL
    assert call(t=None) == EINVAL and call(eps=0.0) == EINVAL
    assert call(bits=16) == EUNSUPPORTED and call(gt=3) == EUNSUPPORTED


def test_the_binding_refuses_tensors_that_are_not_on_the_gpu():
    import torch
    import paper_1907_10134_amd as bp
    x, w, n = torch.zeros(4, 2, 8), torch.zeros(8, 4), torch.zeros(4, 2, 1, 4)
    with pytest.raises(ValueError, match="GPU"):
        bp.ssm_conv(x, w)
    with pytest.raises(ValueError, match="GPU"):
        bp.ssm_scan(x, x, torch.zeros(8, 4), n, n)
    with pytest.raises(ValueError, match=r"\[T, B, D\]"):
        bp.ssm_scan(x[0], x, torch.zeros(8, 4), n, n)
    with pytest.raises(ValueError, match="float32, bfloat16 or float16"):
        bp.ssm_conv(x.double(), w)
    with pytest.raises(TypeError):
        bp.ssm_conv(None, w)
    with pytest.raises(ValueError, match="state_bits"):
        bp.AdamW([w], [w], state_bits=16)
    with pytest.raises(ValueError, match="as many gradients"):
        bp.AdamW([w], [])
    with pytest.raises(ValueError, match="GPU"):
        bp.AdamW([w], [w])
