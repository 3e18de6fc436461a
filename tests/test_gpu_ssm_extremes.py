"""GPU: the state space layer where values are at the ends of their types."""
import numpy as np
import pytest

from oracle import ssm
from test_gpu_ssm import _act, _case, _close, _f64

pytestmark = pytest.mark.gpu


def _lowest(dtype):
    import torch
    return float(torch.finfo(getattr(torch, dtype)).min)


@pytest.mark.parametrize("dtype", ("float32", "bfloat16", "float16"))
def test_gates_of_large_negative_values(dtype):
    """silu and its derivative are zero there: the lowest value of a type is what a mask is filled with."""
    import torch
    import paper_1907_10134_amd as bp
    T, B, D, N = 24, 2, 70, 16
    c, _, dy, dy_ref = _case(21, T, B, D, N, 1, dtype, True, True, False, "tb")
    low = _lowest(dtype)
    c["z"][:, 0, ::3] = low
    c["z"][::2, 1, 1::3] = max(low, -1e30)
    c["z"][5, 1] = max(low, -90.0)
    ref = {k: _f64(v) for k, v in c.items()}
    states = bp.ssm_scan_states(T, B, D, N)
    y = bp.ssm_scan(**c, states=states)
    y_ref = ssm.scan(**ref)[0]
    assert np.all(np.abs(y_ref[:, 0, ::3]) == 0)
    _close(y, y_ref, dtype, "y", sums=N + 2)
    g = bp.ssm_scan_backward(dy, states=states, **c)
    want = ssm.scan_backward(dy_ref, **ref)
    for name in ("du", "ddt", "dz"):
        _close(getattr(g, name), want[name], dtype, name, sums=2 * N + 8)
    for name in ("dBm", "dCm"):
        _close(getattr(g, name), want[name], dtype, name, sums=66)
    one = {k: v[0] if k in ("u", "dt", "z", "Bm", "Cm") else v for k, v in c.items() if k != "h0"}
    state = c["h0"].clone()
    _close(bp.ssm_scan_step(state=state, **one), y_ref[0], dtype, "the token's y", sums=N + 2)


@pytest.mark.parametrize("dtype", ("float32", "bfloat16", "float16"))
@pytest.mark.parametrize("size", (-1e30, None))
def test_convolutions_of_large_negative_values(dtype, size):
    """With weights of one sign p is as large and negative as the input: y is zero, and so is what comes back through it."""
    import torch
    import paper_1907_10134_amd as bp
    T, B, D, W = 70, 2, 41, 4
    rng = np.random.default_rng(4)
    x, dy = _act(rng, (T, B, D), dtype), _act(rng, (T, B, D), dtype)
    low = _lowest(dtype)
    x[3::9, :, ::2] = low if size is None else max(low, size)
    w = torch.from_numpy(rng.uniform(0.1, 0.9, (D, W)).astype(np.float32)).cuda()
    y_ref, _, p, _ = ssm.conv(_f64(x), _f64(w))
    assert float(np.min(p)) < -6000
    _close(bp.ssm_conv(x, w), y_ref, dtype, "y")
    want = ssm.conv_backward(_f64(dy), _f64(x), _f64(w))
    _close(bp.ssm_conv_backward(dy, x, w).dx, want["dx"], dtype, "dx")
    state = x[:W - 1].transpose(0, 1).contiguous()
    _close(bp.ssm_conv_step(x[W - 1], w, None, state), y_ref[W - 1], dtype, "the token's y")


def test_states_that_grow_from_small_ones():
    """A positive A: over the second of three spans of 32 steps a state of 1e-30 grows by e^93, further than the largest float is from
    one, and so does the gradient on its way back.  The exponent, 32 steps times A, is off by a rounding each of the step's size (of
    two, 2^-23), A log2(e), their product and the steps' sum: 93 * 2.5 * 2^-23 = 2.8e-5 of the result; 64 other steps add 2^-23 each."""
    import torch
    import paper_1907_10134_amd as bp
    T, B, D, N = 96, 1, 64, 16
    c, _, dy, _ = _case(13, T, B, D, N, 1, "float32", False, False, False, "tb")
    c["A"].fill_(2.0)
    c["dt"].fill_(-20.0)
    c["dt"][32:64] = 1.19                                # softplus: 1.455
    c["u"].zero_()
    c["h0"] = torch.full((B, D, N), 1e-30, device="cuda") * (1 + torch.rand((B, D, N), device="cuda"))
    dy[:64] = 0.0
    dy[64:] *= 1e-30
    ref = {k: _f64(v) for k, v in c.items()}
    states, h_last = bp.ssm_scan_states(T, B, D, N), torch.empty((B, D, N), device="cuda")
    off = lambda got, want, what: np.testing.assert_allclose(_f64(got), want, rtol=0, atol=4e-5 * np.max(np.abs(want)), err_msg=what)
    y_ref, last_ref, _, _ = ssm.scan(**ref)
    assert 1e9 < np.max(last_ref) < 1e13
    y = bp.ssm_scan(**c, h_last=h_last, states=states)
    off(h_last, last_ref, "h_last")
    off(y, y_ref, "y")
    dh0 = torch.empty((B, D, N), device="cuda")
    g = bp.ssm_scan_backward(dy, states=states, dh0=dh0, **c)
    want = ssm.scan_backward(_f64(dy), **ref)
    assert np.max(np.abs(want["dh0"])) > 1e8
    off(dh0, want["dh0"], "dh0")
    off(g.du[:32], want["du"][:32], "du")


def test_sums_over_many_steps_in_one_span():
    """Gradients of parameters where samples fill the device and time is one span of 65536 steps, all terms alike: single sums in 32 bits
    would be off by up to 65536 roundings of half a step each in the same direction.  Held: 512 steps in a row, their 128
    sums, then the samples, a quarter each: (512 + 128 + 513 + 3) 2^-24 at the most, and a step's own terms, of which
    exp, softplus, products and sums of two states are good to some 2^-21 each with the memory of 1 / (1 - 0.61) steps."""
    import torch
    import paper_1907_10134_amd as bp
    T, B = 1 << 16, 2049
    all_ = lambda x, *shape: torch.full((1,) * len(shape), x, device="cuda").expand(shape)
    c = {"u": all_(1.1, T, B, 1), "dt": all_(0.3, T, B, 1), "Bm": all_(0.7, T, B, 1, 1), "Cm": all_(0.9, T, B, 1, 1),
         "A": torch.full((1, 1), -0.57, device="cuda"), "skip": torch.full((1,), 0.37, device="cuda"),
         "dt_bias": torch.zeros(1, device="cuda")}
    dy = all_(0.77, T, B, 1)
    states = bp.ssm_scan_states(T, B, 1, 1)
    bp.ssm_scan(**c, states=states)
    g = bp.ssm_scan_backward(dy, states=states, **c)
    one = lambda x: _f64(x[:, :1]) if x.dim() > 2 else _f64(x)
    want = ssm.scan_backward(_f64(dy[:, :1]), **{k: one(v) for k, v in c.items()})
    for name in ("dA", "dskip", "ddt_bias"):
        off = abs(float(getattr(g, name)) / (float(want[name].item()) * B) - 1)
        assert off <= 1156 * 2.0 ** -24 + 2 * 2.0 ** -21, (name, off)


@pytest.mark.parametrize("way", ("time", "samples"))
def test_windows_of_one_array_as_inputs(way):
    """Rows that overlap, [t] or [b] one element behind the last: the gradients come back with their channels side by side."""
    import torch
    import paper_1907_10134_amd as bp
    T, B, D, N = 12, 3, 20, 8
    c, _, dy, dy_ref = _case(14, T, B, D, N, 1, "float32", True, True, False, "tb")
    of = lambda x: x.as_strided((T, B, D), (1, 40, 1) if way == "time" else (40, 1, 1))
    for name in ("u", "dt", "z"):
        c[name] = of(c[name].contiguous().flatten())
    ref = {k: _f64(v) for k, v in c.items()}
    states = bp.ssm_scan_states(T, B, D, N)
    _close(bp.ssm_scan(**c, states=states), ssm.scan(**ref)[0], "float32", "y", sums=N + 2)
    g = bp.ssm_scan_backward(dy, states=states, **c)
    want = ssm.scan_backward(dy_ref, **ref)
    for name in ("du", "ddt", "dz"):
        _close(getattr(g, name), want[name], "float32", name, sums=2 * N + 8)
    w = torch.rand((D, 4), device="cuda") - 0.5
    _close(bp.ssm_conv(c["u"], w), ssm.conv(ref["u"], _f64(w))[0], "float32", "conv")
    _close(bp.ssm_conv_backward(dy, c["u"], w).dx, ssm.conv_backward(dy_ref, ref["u"], _f64(w))["dx"], "float32", "dx")


@pytest.mark.parametrize("N", (49, 64))
@pytest.mark.parametrize("dtype", ("float32", "bfloat16"))
@pytest.mark.parametrize("gate,given,ragged", [(False, True, False), (True, True, True)])
def test_sixteen_waves_and_many_spans(N, dtype, gate, given, ragged):
    """The widest workgroups with time in spans: their summaries and joins."""
    from test_gpu_ssm import test_scan_and_gradients as whole
    whole((1100, 2, 40, N, 1), dtype, gate, given, ragged, "bt")


@pytest.mark.parametrize("T", (504, 513, 520, 1032))
@pytest.mark.parametrize("N,gate", [(1, True), (20, False)])
def test_sums_in_runs_of_512_steps(T, N, gate):
    """One span of 63 to 129 passes of eight steps, ragged: the runs' ends, a sample that ends inside one and an empty one."""
    import torch
    import paper_1907_10134_amd as bp
    B = 4100 if N == 1 else 1040                         # samples enough for the device without spans of time
    c, ref, dy, dy_ref = _case(T, T, B, 1, N, 1, "float32", gate, True, True, "tb")
    c["lengths"][1], c["lengths"][2], c["lengths"][3] = T, min(T, 513), min(T, 520)
    for k in ("u", "dt", "Bm", "Cm") + (("z",) if gate else ()):
        c[k].nan_to_num_(nan=0.25)
    dy.nan_to_num_(nan=0.25)
    ref = {k: _f64(v) for k, v in c.items()}
    states, dh0 = bp.ssm_scan_states(T, B, 1, N), torch.empty((B, 1, N), device="cuda")
    bp.ssm_scan(**c, states=states)
    g = bp.ssm_scan_backward(dy, states=states, dh0=dh0, **c)
    want = ssm.scan_backward(_f64(dy), **ref)
    along = 512 + T // 512 + B // 4                      # a run, the runs, a quarter of the samples
    for name in ("dA", "dskip", "ddt_bias"):
        _close(getattr(g, name), want[name], "float32", name, sums=along)
    _close(dh0, want["dh0"], "float32", "dh0")
