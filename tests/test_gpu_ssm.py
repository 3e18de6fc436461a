"""GPU: the state space layer's operators against the fp64 oracle."""
import numpy as np
import pytest

from oracle import ssm

pytestmark = pytest.mark.gpu

TYPES = ("float32", "bfloat16", "float16")


def _bound(ref, dtype, sums):
    """Half a step of the output's type relative to the value, and fp32 arithmetic relative to the largest of the tensor:
    an error of 2^-23 a step (exp and softplus are good to that, products and sums to half of it) kept over a state's memory of
    at most 100 steps here, 1.2e-5, and `sums` of so many fp32 parts in a row, 2^-24 of the largest each."""
    import torch
    half = torch.finfo(getattr(torch, dtype)).eps / 2
    return half * np.abs(ref) + (100 * 2.0 ** -23 + sums * 2.0 ** -24) * max(np.max(np.abs(ref), initial=0.0), 2.0 ** -14)


def _close(got, ref, dtype, what, sums=16):
    got = got.detach().double().cpu().numpy()
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    off = np.abs(got - ref)
    assert np.all(np.isfinite(got)), what
    worst = np.max(off - _bound(ref, dtype, sums), initial=0.0)
    assert worst <= 0, (what, float(np.max(off)), float(np.max(np.abs(ref), initial=0.0)))


def _act(rng, shape, dtype, order="tb", wide=0, at=0, scale=1.0):
    """A tensor [T, B, C] on the GPU, as a column slice of a wider one if `wide`, with the values that it then holds."""
    import torch
    T, B, C = shape
    full = (B, T, wide or C) if order == "bt" else (T, B, wide or C)
    x = torch.from_numpy(rng.standard_normal(full) * scale).to(getattr(torch, dtype)).cuda()
    if order == "bt":
        x = x.transpose(0, 1)
    return x[:, :, at:at + C]


def _f64(x):
    return x.detach().double().cpu().numpy()


def _case(seed, T, B, D, N, G, dtype, gate, given, ragged, order):
    import torch
    rng = np.random.default_rng(seed)
    f32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda()
    c = {"u": _act(rng, (T, B, D), dtype, order), "dt": _act(rng, (T, B, D), dtype, order, scale=0.5),
         "A": f32(-rng.uniform(0.2, 4.0, (D, N)))}
    proj = _act(rng, (T, B, 2 * G * N + 3), dtype, order)
    c["Bm"] = proj[:, :, 3:3 + G * N].unflatten(2, (G, N))
    c["Cm"] = proj[:, :, 3 + G * N:].unflatten(2, (G, N))
    if gate:
        c["z"] = _act(rng, (T, B, D), dtype, order, wide=2 * D + 1, at=D)
    if given:
        c.update(skip=f32(rng.standard_normal(D)), dt_bias=f32(rng.uniform(-3.0, 0.0, D)), h0=f32(rng.standard_normal((B, D, N))))
    dy = _act(rng, (T, B, D), dtype, order)
    if ragged:
        n = rng.integers(0, T + 1, B)
        n[0] = T // 2
        n[-1] = 0 if B > 1 else 1
        c["lengths"] = torch.from_numpy(n.astype(np.int32)).cuda()
    ref = {k: _f64(v) for k, v in c.items()}
    dy_ref = _f64(dy)
    if ragged:                                 # what lies behind a sample's end must not be read: NaN there
        for b, k in enumerate(ref["lengths"].astype(int)):
            for name in ("u", "dt", "Bm", "Cm") + (("z",) if gate else ()):
                c[name][k:, b] = float("nan")
                ref[name][k:, b] = 0.0
            dy[k:, b] = float("nan")
            dy_ref[k:, b] = 0.0
    return c, ref, dy, dy_ref


SIZES = [(1, 1, 1, 1, 1), (2, 3, 5, 3, 1), (7, 1, 64, 4, 1), (8, 2, 65, 8, 1), (9, 2, 70, 16, 2), (17, 4, 130, 16, 1),
         (64, 3, 66, 5, 3), (130, 2, 20, 24, 1), (40, 2, 64, 64, 1), (33, 2, 48, 33, 2), (257, 1, 129, 16, 1), (1000, 2, 40, 16, 1),
         (700, 1, 320, 4, 5), (2111, 1, 33, 12, 1), (515, 3, 8, 32, 4), (300, 2, 128, 48, 2)]


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gate,given,ragged,order", [(False, False, False, "tb"), (True, True, False, "bt"),
                                                     (True, False, True, "tb"), (False, True, True, "bt")])
def test_scan_and_gradients(size, dtype, gate, given, ragged, order):
    import torch
    import paper_1907_10134_amd as bp
    T, B, D, N, G = size
    c, ref, dy, dy_ref = _case(sum(size) + len(dtype), T, B, D, N, G, dtype, gate, given, ragged, order)
    y_ref, last_ref, _, _ = ssm.scan(**ref)
    h_last = torch.full((B, D, N), float("nan"), device="cuda")
    y = bp.ssm_scan(**c, h_last=h_last)
    _close(y, y_ref, dtype, "y", sums=N + 2)
    _close(h_last, last_ref, "float32", "h_last")
    states = bp.ssm_scan_states(T, B, D, N)
    y2 = bp.ssm_scan(**c, states=states)
    _close(y2, y_ref, dtype, "y with states", sums=N + 2)
    dh0 = torch.full((B, D, N), float("nan"), device="cuda")
    g = bp.ssm_scan_backward(dy, states=states, dh0=dh0, **c)
    want = ssm.scan_backward(dy_ref, **ref)
    along = 64 + T * B // 64                   # sums over time and samples: 64 in a row at most, then their totals
    for name in ("du", "ddt") + (("dz",) if gate else ()):
        _close(getattr(g, name), want[name], dtype, name, sums=2 * N + 8)
    for name in ("dBm", "dCm"):
        _close(getattr(g, name), want[name], dtype, name, sums=64 + D // 64)
    _close(g.dA, want["dA"], "float32", "dA", sums=along)
    _close(dh0, want["dh0"], "float32", "dh0")
    assert (g.dskip is None) == (not given) and (g.ddt_bias is None) == (not given) and (g.dz is None) == (not gate)
    if given:
        _close(g.dskip, want["dskip"], "float32", "dskip", sums=along)
        _close(g.ddt_bias, want["ddt_bias"], "float32", "ddt_bias", sums=along)
    again = bp.ssm_scan_backward(dy, states=states, dh0=torch.empty_like(dh0), **c)
    assert all(torch.equal(a, b) for a, b in zip(g[:8], again[:8]) if a is not None), "the same bits on every call"
    assert torch.equal(y2, bp.ssm_scan(**c, states=states))


def test_scan_gradients_against_differences():
    """dA, dh0 and du of the kernels against central differences of the kernels' own forward pass, float32: the loss is a sum
    of 6144 terms of order one, good to 1e-6 of its 100 or so, over 2e-2: 1e-2 of the largest gradient."""
    import torch
    import paper_1907_10134_amd as bp
    T, B, D, N, G = 96, 2, 32, 8, 1
    c, _, dy, _ = _case(11, T, B, D, N, G, "float32", True, True, False, "tb")
    states = bp.ssm_scan_states(T, B, D, N)
    bp.ssm_scan(**c, states=states)
    g = bp.ssm_scan_backward(dy, states=states, dh0=torch.empty((B, D, N), device="cuda"), **c)
    loss = lambda: float((bp.ssm_scan(**c).double() * dy.double()).sum())
    for name, grad in (("A", g.dA), ("h0", g.dh0), ("u", g.du), ("dt", g.ddt), ("skip", g.dskip), ("dt_bias", g.ddt_bias)):
        flat, at = c[name].view(-1), int(grad.abs().argmax())
        was = float(flat[at])
        flat[at] = was + 1e-2
        up = loss()
        flat[at] = was - 1e-2
        down = loss()
        flat[at] = was
        want = float(grad.view(-1)[at])
        assert abs((up - down) / 2e-2 - want) <= 1e-2 * abs(want) + 1e-2, (name, (up - down) / 2e-2, want)


def test_a_step_that_hardly_moves_and_one_that_forgets():
    """softplus at both ends: steps of e^-15 and of 40, decays of 1 and 0; and an infinite gate input where it says zero."""
    import torch
    import paper_1907_10134_amd as bp
    T, B, D, N = 24, 1, 64, 16
    c, ref, _, _ = _case(5, T, B, D, N, 1, "float32", True, True, False, "tb")
    c["dt"][:, :, ::2] = -15.0
    c["dt"][:, :, 1::4] = 40.0
    c["z"][:, :, 3] = -80.0
    ref = {k: _f64(v) for k, v in c.items()}
    h_last = torch.empty((B, D, N), device="cuda")
    _close(bp.ssm_scan(**c, h_last=h_last), ssm.scan(**ref)[0], "float32", "y", sums=N)
    _close(h_last, ssm.scan(**ref)[1], "float32", "h_last")


def test_states_that_grow():
    """A positive A: nothing enters for 900 steps, over which the decay's product passes the largest float many times, and
    the states of the last steps grow from there; the same for the gradient, from the other end."""
    import torch
    import paper_1907_10134_amd as bp
    T, B, D, N = 910, 1, 64, 16
    c, _, dy, _ = _case(12, T, B, D, N, 1, "float32", False, False, False, "tb")
    c["A"].fill_(2.0)
    c["dt"].fill_(1.0)
    c["u"][:900] = 0.0
    dy[10:] = 0.0
    states = bp.ssm_scan_states(T, B, D, N)
    y = bp.ssm_scan(**c, states=states)
    _close(y, ssm.scan(**{k: _f64(v) for k, v in c.items()})[0], "float32", "y", sums=N)
    g = bp.ssm_scan_backward(dy, states=states, **c)
    assert all(bool(torch.isfinite(x).all()) for x in (g.du, g.ddt, g.dA, g.dBm, g.dCm))
    want = ssm.scan_backward(_f64(dy), **{k: _f64(v) for k, v in c.items()})
    _close(g.du, want["du"], "float32", "du", sums=2 * N)


def test_a_nan_stays_in_its_channel():
    import torch
    import paper_1907_10134_amd as bp
    c, _, _, _ = _case(6, 100, 2, 96, 16, 1, "float32", False, True, False, "tb")
    c["u"][50, 1, 70] = float("nan")
    y = bp.ssm_scan(**c)
    bad = torch.isnan(y)
    assert bool(bad[50:, 1, 70].all()) and int(bad.sum()) == 50


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,D,N,G,gate,slots", [(1, 1, 1, 1, False, 1), (3, 70, 16, 1, True, 9), (5, 64, 5, 2, True, 5),
                                                (2, 130, 64, 1, False, 4), (67, 96, 24, 3, True, 70), (4, 33, 33, 1, False, 8)])
def test_scan_step(dtype, B, D, N, G, gate, slots):
    import torch
    import paper_1907_10134_amd as bp
    c, ref, _, _ = _case(B + D + N, 1, B, D, N, G, dtype, gate, True, False, "tb")
    del c["h0"], ref["h0"]
    rng = np.random.default_rng(1)
    state = torch.from_numpy(rng.standard_normal((slots, D, N)).astype(np.float32)).cuda()
    at = rng.permutation(slots)[:B].astype(np.int32)
    if B > 2:
        at[1], at[2] = -1, slots                  # rows of no stream
    on = (at >= 0) & (at < slots)
    before = _f64(state)
    one = {k: v[0] if k in ("u", "dt", "z", "Bm", "Cm") else v for k, v in c.items()}
    y = bp.ssm_scan_step(state=state, slots=torch.from_numpy(at).cuda(), **one)
    ref["h0"] = np.zeros((B, D, N))
    ref["h0"][on] = before[at[on]]
    y_ref, last, _, _ = ssm.scan(**ref)
    y_ref[0, ~on] = 0.0
    want = before.copy()
    want[at[on]] = last[on]
    _close(y, y_ref[0], dtype, "y", sums=N + 2)
    _close(state, want, "float32", "state")
    untouched = np.setdiff1d(np.arange(slots), at[on])
    assert np.array_equal(_f64(state)[untouched], before[untouched])


CONV_SIZES = [(1, 1, 1, 2), (1, 2, 5, 4), (2, 3, 64, 4), (3, 1, 7, 4), (63, 2, 65, 3), (64, 2, 128, 4), (65, 3, 130, 2), (200, 2, 41, 4),
              (1030, 1, 96, 4), (16, 5, 1024, 3)]


@pytest.mark.parametrize("size", CONV_SIZES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("silu,given,ragged,order,at", [(True, True, False, "tb", 0), (False, False, False, "bt", 1),
                                                        (True, True, True, "bt", 0), (True, False, True, "tb", 3)])
def test_conv_and_gradients(size, dtype, silu, given, ragged, order, at):
    import torch
    import paper_1907_10134_amd as bp
    T, B, D, W = size
    rng = np.random.default_rng(sum(size) + at)
    f32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda()
    x = _act(rng, (T, B, D), dtype, order, wide=2 * D + at, at=at)
    dy = _act(rng, (T, B, D), dtype, order)
    c = {"weight": f32(rng.uniform(-0.5, 0.5, (D, W)))}
    if given:
        c.update(bias=f32(rng.uniform(-0.5, 0.5, D)), state0=_act(rng, (B, W - 1, D), dtype))
    if ragged:
        n = rng.integers(0, T + 1, B)
        n[-1] = 0 if B > 1 else 1
        c["lengths"] = torch.from_numpy(n.astype(np.int32)).cuda()
    ref = {k: _f64(v) for k, v in c.items()}
    x_ref, dy_ref = _f64(x), _f64(dy)
    if ragged:
        for b, k in enumerate(ref["lengths"].astype(int)):
            x[k:, b] = float("nan")
            dy[k:, b] = float("nan")
            x_ref[k:, b] = dy_ref[k:, b] = 0.0
    last = torch.full((B, W - 1, D), float("nan"), dtype=x.dtype, device="cuda")
    y = bp.ssm_conv(x, **c, silu=silu, state_last=last)
    y_ref, last_ref, _, _ = ssm.conv(x_ref, **ref, silu=silu)
    _close(y, y_ref, dtype, "y")
    assert np.array_equal(_f64(last), last_ref)
    d0 = torch.full((B, W - 1, D), float("nan"), dtype=x.dtype, device="cuda")
    g = bp.ssm_conv_backward(dy, x, **c, silu=silu, dstate0=d0)
    want = ssm.conv_backward(dy_ref, x_ref, **ref, silu=silu)
    _close(g.dx, want["dx"], dtype, "dx")
    _close(d0, want["dstate0"], dtype, "dstate0")
    _close(g.dweight, want["dweight"], "float32", "dweight", sums=64 + T * B // 64)
    if given:
        _close(g.dbias, want["dbias"], "float32", "dbias", sums=64 + T * B // 64)
    again = bp.ssm_conv_backward(dy, x, **c, silu=silu, dstate0=torch.empty_like(d0))
    assert torch.equal(g.dweight, again.dweight) and torch.equal(g.dx, again.dx)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,D,W,silu", [(1, 1, 2, True), (3, 70, 4, True), (5, 64, 3, False), (66, 257, 4, True), (4, 512, 4, True)])
def test_conv_step(dtype, B, D, W, silu):
    import torch
    import paper_1907_10134_amd as bp
    rng = np.random.default_rng(B + D)
    slots = B + 3
    x = _act(rng, (1, B, D), dtype, wide=2 * D)[0]
    state = _act(rng, (slots, W - 1, D), dtype).contiguous()
    w = torch.from_numpy(rng.uniform(-0.5, 0.5, (D, W)).astype(np.float32)).cuda()
    bias = torch.from_numpy(rng.uniform(-0.5, 0.5, D).astype(np.float32)).cuda()
    at = rng.permutation(slots)[:B].astype(np.int32)
    if B > 2:
        at[0], at[2] = -1, slots + 5
    on = (at >= 0) & (at < slots)
    before, x_ref = _f64(state), _f64(x)
    y = bp.ssm_conv_step(x, w, bias, state, silu=silu, slots=torch.from_numpy(at).cuda())
    y_ref, last, _, _ = ssm.conv(x_ref[None][:, on], _f64(w), _f64(bias), silu, before[at[on]])
    want_y = np.zeros((B, D))
    want_y[on] = y_ref[0]
    _close(y, want_y, dtype, "y")
    want = before.copy()
    want[at[on]] = last
    assert np.array_equal(_f64(state), want)


def test_rows_further_apart_than_32_bits_count():
    """Rows 2^28 elements apart, nine of them: the last lies 2^31 elements behind the first."""
    import torch
    import paper_1907_10134_amd as bp
    rng = np.random.default_rng(2)
    T, D, N = 9, 64, 16
    wide = torch.empty((T, 1, 1 << 28), dtype=torch.bfloat16, device="cuda")
    put = lambda at, c: wide[:, :, at:at + c].copy_(_act(rng, (T, 1, c), "bfloat16"))
    u, dt, bm, cm, dy = put(0, D), put(64, D), put(128, N), put(144, N), put(192, D)
    A = -torch.rand((D, N), device="cuda") - 0.1
    w = torch.rand((D, 4), device="cuda") - 0.5
    bm, cm = bm.unflatten(2, (1, N)), cm.unflatten(2, (1, N))
    out = wide[:, :, 256:320]
    states = bp.ssm_scan_states(T, 1, D, N)
    bp.ssm_scan(u, dt, A, bm, cm, y=out, states=states)
    ref = dict(u=_f64(u), dt=_f64(dt), A=_f64(A), Bm=_f64(bm), Cm=_f64(cm))
    _close(out, ssm.scan(**ref)[0], "bfloat16", "y", sums=N)
    g = bp.ssm_scan_backward(dy, u, dt, A, bm, cm, states)
    want = ssm.scan_backward(_f64(dy), **ref)
    _close(g.du, want["du"], "bfloat16", "du", sums=40)
    _close(g.dA, want["dA"], "float32", "dA", sums=64)
    bp.ssm_conv(u, w, y=out)
    _close(out, ssm.conv(ref["u"], _f64(w))[0], "bfloat16", "conv")
    _close(bp.ssm_conv_backward(dy, u, w).dx, ssm.conv_backward(_f64(dy), ref["u"], _f64(w))["dx"], "bfloat16", "dx")


def test_more_tokens_than_one_round_of_the_joining_launch_has():
    """2^25 tokens of a channel and a state, 2^29 places of dB and dC: the first, a middle and the last sample's."""
    import torch
    import paper_1907_10134_amd as bp
    T, B = 1 << 14, 2048
    torch.manual_seed(3)
    r = lambda *shape: torch.randn(shape, device="cuda")
    u, dt, bm, cm, dy = r(T, B, 1), 0.5 * r(T, B, 1), r(T, B, 1, 1), r(T, B, 1, 1), r(T, B, 1)
    A = torch.full((1, 1), -1.0, device="cuda")
    states = bp.ssm_scan_states(T, B, 1, 1)
    y = bp.ssm_scan(u, dt, A, bm, cm, states=states)
    g = bp.ssm_scan_backward(dy, u, dt, A, bm, cm, states)
    for b in (0, 1000, B - 1):
        at = slice(b, b + 1)
        ref = dict(u=_f64(u[:, at]), dt=_f64(dt[:, at]), A=_f64(A), Bm=_f64(bm[:, at]), Cm=_f64(cm[:, at]))
        _close(y[:, at], ssm.scan(**ref)[0], "float32", "y", sums=3)
        want = ssm.scan_backward(_f64(dy[:, at]), **ref)
        for name in ("du", "ddt", "dBm", "dCm"):
            _close(getattr(g, name)[:, at], want[name], "float32", name, sums=65)


def test_inputs_that_repeat_a_row():
    """Broadcast inputs, strides of zero: read as they say; the gradient is that of each place."""
    import torch
    import paper_1907_10134_amd as bp
    c, ref, dy, dy_ref = _case(8, 20, 3, 40, 8, 1, "float32", False, False, False, "tb")
    c["u"] = c["u"][:1].expand(20, 3, 40)
    c["Bm"] = c["Bm"][:, :1].expand(20, 3, 1, 8)
    ref["u"], ref["Bm"] = _f64(c["u"]), _f64(c["Bm"])
    states = bp.ssm_scan_states(20, 3, 40, 8)
    _close(bp.ssm_scan(**c, states=states), ssm.scan(**ref)[0], "float32", "y", sums=10)
    g = bp.ssm_scan_backward(dy, states=states, **c)
    want = ssm.scan_backward(dy_ref, **ref)
    _close(g.du, want["du"], "float32", "du", sums=24)
    _close(g.dBm, want["dBm"], "float32", "dBm", sums=64)
    with pytest.raises(bp.BppsaError):
        bp.ssm_scan(**c, y=torch.empty((1, 3, 40), device="cuda").expand(20, 3, 40))


def test_another_stream_and_a_graph():
    """The training calls on a stream of their own, then captured and replayed between eager calls: the eager bits each time."""
    import torch
    import paper_1907_10134_amd as bp
    T, B, D, N = 300, 2, 96, 16
    c, _, dy, _ = _case(9, T, B, D, N, 1, "bfloat16", True, True, True, "tb")
    w = torch.rand((D, 4), device="cuda") - 0.5
    states, dh0 = bp.ssm_scan_states(T, B, D, N), torch.empty((B, D, N), device="cuda")
    n = c["lengths"]

    def work(stream=None):
        y = bp.ssm_scan(**c, states=states, stream=stream)
        g = bp.ssm_scan_backward(dy, states=states, dh0=dh0, stream=stream, **c)
        h = bp.ssm_conv(c["u"], w, lengths=n, stream=stream)
        k = bp.ssm_conv_backward(dy, c["u"], w, lengths=n, stream=stream)
        return [y, *(x for x in g if x is not None), h, k.dx, k.dweight]

    want = [x.clone() for x in work()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = work(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = work()
    for _ in range(4):
        for x in held:
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want))
        assert all(torch.equal(a, b) for a, b in zip(work(), want))


def test_refusals():
    import torch
    import paper_1907_10134_amd as bp
    c, _, dy, _ = _case(10, 8, 2, 16, 4, 2, "float32", False, True, False, "tb")
    bad = lambda **k: pytest.raises(ValueError, bp.ssm_scan, **dict(c, **k))
    bad(u=c["u"].double())
    bad(dt=c["dt"].half())
    bad(dt=c["dt"][:4])
    bad(Bm=c["Bm"].transpose(2, 3).contiguous().transpose(2, 3))
    bad(A=c["A"].t().contiguous().t())
    bad(A=c["A"][:8])
    bad(h0=c["h0"][:1])
    bad(lengths=torch.ones(2, dtype=torch.int64, device="cuda"))
    bad(lengths=torch.ones(3, dtype=torch.int32, device="cuda"))
    bad(states=torch.empty(8, dtype=torch.uint8, device="cuda"))
    bad(u=torch.empty((8, 2, 32), device="cuda")[:, :, ::2])
    with pytest.raises(bp.BppsaError):
        bp.ssm_scan(c["u"][:0], c["dt"][:0], c["A"], c["Bm"][:0], c["Cm"][:0])
    with pytest.raises(bp.BppsaError):
        bp.ssm_scan(**dict(c, Bm=c["Bm"].expand(8, 2, 2, 4)[:, :, :1].expand(8, 2, 3, 4).contiguous(),
                           Cm=c["Cm"][:, :, :1].expand(8, 2, 3, 4).contiguous()))      # 16 channels, 3 groups
    with pytest.raises(TypeError):
        bp.ssm_scan_backward(dy, c["u"], c["dt"], c["A"], c["Bm"], c["Cm"], None)
    with pytest.raises(ValueError):
        bp.ssm_scan_step(c["u"][0], c["dt"][0], c["A"], c["Bm"][0], c["Cm"][0], torch.empty((1, 16, 4), device="cuda"))
    with pytest.raises(ValueError):
        bp.ssm_conv_step(c["u"][0], torch.empty((16, 4), device="cuda"), None, torch.empty((4, 2, 16), device="cuda"))
    with pytest.raises(bp.BppsaError):
        bp.ssm_conv(c["u"], torch.empty((16, 7), device="cuda"))
