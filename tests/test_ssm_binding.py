"""The state space layer's binding: streams of the caller's choice, and what it refuses."""
import contextlib

import pytest


class _Made:
    def __init__(self):
        self.recorded = []

    def record_stream(self, stream):
        self.recorded.append(stream)


class _Stream:
    device = "cuda:0"


def test_what_a_call_makes_on_another_stream_is_that_streams(monkeypatch):
    """Allocated with the stream current, and kept from it until the caller's stream is done: every array of every result."""
    import torch
    from paper_1907_10134_amd import ssm
    here, side, now = _Stream(), _Stream(), []

    @contextlib.contextmanager
    def on(stream):
        now.append(stream)
        yield
        now.pop()

    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: now[-1] if now else here)

    def call(make):
        assert torch.cuda.current_stream() is side
        return make()

    one = ssm._aside(side, call, _Made)
    assert one.recorded == [here] and not now
    g = ssm._aside(side, call, lambda: ssm.SsmGrads(*([_Made() for _ in range(8)] + [None])))
    assert type(g) is ssm.SsmGrads and g.dh0 is None and all(x.recorded == [here] for x in g[:8])
    now.append(side)                           # already the current one
    assert ssm._aside(side, call, _Made).recorded == []


@pytest.mark.parametrize("name", ("ssm_scan", "ssm_scan_backward", "ssm_scan_step", "ssm_conv", "ssm_conv_backward", "ssm_conv_step"))
def test_every_call_hands_all_its_arguments_over(monkeypatch, name):
    import inspect
    from paper_1907_10134_amd import ssm
    call, got = getattr(ssm, name), []
    monkeypatch.setattr(ssm, "_aside", lambda stream, again, *args: got.append((stream, again, args)))
    names = [k for k in inspect.signature(call).parameters if k != "stream"]
    assert list(inspect.signature(call).parameters)[-1] == "stream"
    call(**{k: k for k in names}, stream="side")
    assert got == [("side", call, tuple(names))]


@pytest.mark.gpu
def test_memory_of_results_on_another_stream_is_not_given_out_again():
    """One field of the result is kept: the others' memory, still being written there, must not become new arrays here."""
    import torch
    import paper_1907_10134_amd as bp
    T, B, D, N = 512, 4, 256, 16
    r = lambda *shape: torch.randn(shape, device="cuda")
    u, dt, z, dy, Bm, Cm, A = r(T, B, D), r(T, B, D), r(T, B, D), r(T, B, D), r(T, B, 1, N), r(T, B, 1, N), -torch.rand((D, N), device="cuda")
    w, bias, one = torch.rand((D, 4), device="cuda") - 0.5, torch.rand(D, device="cuda"), torch.ones(D, device="cuda")
    states = bp.ssm_scan_states(T, B, D, N)
    call = lambda stream: (bp.ssm_scan(u, dt, A, Bm, Cm, one, z, bias, states=states, stream=stream),
                           *bp.ssm_scan_backward(dy, u, dt, A, Bm, Cm, states, one, z, bias, stream=stream)[:8],
                           bp.ssm_conv(u, w, bias, stream=stream), *bp.ssm_conv_backward(dy, u, w, bias, stream=stream)[:3],
                           bp.ssm_scan_step(u[0], dt[0], A, Bm[0], Cm[0], torch.zeros((B, D, N), device="cuda"), stream=stream),
                           bp.ssm_conv_step(u[0], w, bias, torch.zeros((B, 3, D), device="cuda"), stream=stream))
    want = call(None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = call(side)
    shapes, places = [x.shape for x in got], {x.data_ptr() for x in got}
    kept = got[1]
    del got
    new = [torch.empty(shape, device="cuda") for shape in shapes for _ in range(2)]
    assert not places & {x.data_ptr() for x in new}
    side.synchronize()
    assert torch.equal(kept, want[1])
    for a, b in zip(call(side), want):
        side.synchronize()
        assert torch.equal(a, b)


def test_a_current_device_that_is_not_the_tensors_is_refused(monkeypatch):
    import torch
    import paper_1907_10134_amd as bp
    from paper_1907_10134_amd import ssm
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    monkeypatch.setattr(ssm, "_current_device", lambda: 1)
    with pytest.raises(ValueError, match="cuda:0, the current device is cuda:1"):
        ssm._here(0)
    opt = object.__new__(bp.AdamW)             # no GPU is needed to be refused
    opt._device, opt.t = 0, 0
    with pytest.raises(ValueError, match="cuda:0"):
        opt.step()
    _Stream.device, was = torch.device("cuda:2"), _Stream.device
    try:
        with pytest.raises(ValueError, match="cuda:2"):
            opt.step(stream=_Stream())
    finally:
        _Stream.device = was
    assert opt.t == 0


@pytest.mark.gpu
def test_tensors_of_several_devices_are_refused(monkeypatch):
    import torch
    import paper_1907_10134_amd as bp
    from paper_1907_10134_amd import ssm
    x, w = torch.zeros((4, 2, 8), device="cuda"), torch.zeros((8, 4), device="cuda")
    for check in (lambda: ssm._rows(x, x.shape, x.dtype, "dt", 1), lambda: ssm._param(w, w.shape, "A", 1),
                  lambda: ssm._token(x[0], x[0].shape, x.dtype, "u", 1), lambda: ssm._on(x, 1, "states")):
        with pytest.raises(ValueError, match="cuda:1 like the first argument"):
            check()
    n = torch.zeros((4, 2, 1, 4), device="cuda")
    for cpu in ("dt", "A", "Bm", "Cm", "skip", "z", "dt_bias", "h0", "lengths", "y", "h_last", "states"):
        c = {"u": x, "dt": x, "A": w, "Bm": n, "Cm": n, "skip": w[:, 0].contiguous(), "z": x, "dt_bias": w[:, 0].contiguous(),
             "h0": torch.zeros((2, 8, 4), device="cuda"), "lengths": torch.ones(2, dtype=torch.int32, device="cuda"),
             "y": torch.empty_like(x), "h_last": torch.zeros((2, 8, 4), device="cuda"), "states": bp.ssm_scan_states(4, 2, 8, 4)}
        c[cpu] = c[cpu].cpu()
        with pytest.raises(ValueError, match="%s must live on the GPU" % cpu):
            bp.ssm_scan(**c)
    with pytest.raises(ValueError, match="state must live on the GPU"):
        bp.ssm_scan_step(x[0], x[0], w, n[0], n[0], torch.zeros((2, 8, 4)))
    with pytest.raises(TypeError):
        bp.ssm_conv_step(x[0], w, None, None)
    with pytest.raises(ValueError, match=r"\[B, D\] and Bm"):
        bp.ssm_scan_step(x, x[0], w, n[0], n[0], torch.zeros((2, 8, 4), device="cuda"))
    with pytest.raises(ValueError, match="Cm must have shape"):
        bp.ssm_scan_step(x[0], x[0], w, n[0], n[0, :1], torch.zeros((2, 8, 4), device="cuda"))
    monkeypatch.setattr(ssm, "_current_device", lambda: 1)
    with pytest.raises(ValueError, match="current device is cuda:1"):
        bp.ssm_conv(x, w)


def test_kept_states_off_16_bytes_are_refused():
    """The kernels read and write them by 8 and 16 bytes."""
    import ctypes
    from test_oracle_ssm import EINVAL, EWORKSPACE, ONE, Grads, Rows, _rows, _ssm
    import paper_1907_10134_amd as bp
    from paper_1907_10134_amd import ssm
    lib = ctypes.CDLL(bp.binding.lib_path())
    p, n = ctypes.c_void_p, ctypes.c_size_t
    need = ssm.ssm_scan_workspace_bytes(4000, 1, 32, 16, 1)
    assert need                                # so that a call with good states ends at the missing workspace
    g = Grads(_rows(), _rows(), Rows(), ONE, ONE, ONE, None, None, None)
    for states, want in ((ONE + 8, EINVAL), (ONE + 1, EINVAL), (ONE + 16, EWORKSPACE)):
        l = ctypes.byref(_ssm(T=4000, B=1))
        assert lib.bppsa_ssm_scan(l, ctypes.byref(_rows()), None, p(states), None, n(0), None) == want
        assert lib.bppsa_ssm_scan_backward(l, ctypes.byref(_rows()), p(states), ctypes.byref(g), None, n(0), None) == want


def test_a_workspace_that_is_not_the_gpus_is_refused():
    import torch
    from paper_1907_10134_amd import ssm
    with pytest.raises(ValueError, match="workspace must live on the GPU"):
        ssm._opaque(torch.empty(1 << 20, dtype=torch.uint8), 4096, 0)
    with pytest.raises(TypeError, match="workspace"):
        ssm._opaque(1 << 20, 4096, 0)


@pytest.mark.gpu
def test_a_workspace_with_gaps_is_refused():
    import torch
    import paper_1907_10134_amd as bp
    from paper_1907_10134_amd import ssm
    T, D, N = 4000, 32, 16
    r = lambda *shape: torch.randn(shape, device="cuda")
    u, dt, Bm, Cm, A = r(T, 1, D), r(T, 1, D), r(T, 1, 1, N), r(T, 1, 1, N), -torch.rand((D, N), device="cuda")
    need = ssm.ssm_scan_workspace_bytes(T, 1, D, N, 1)
    for bad in (torch.empty((need, 2), dtype=torch.uint8, device="cuda")[:, 0], torch.empty(4, device="cuda").expand(need, 4)):
        with pytest.raises(ValueError, match="workspace must be contiguous"):
            bp.ssm_scan(u, dt, A, Bm, Cm, workspace=bad)
    with pytest.raises(bp.BppsaError):
        bp.ssm_scan(u, dt, A, Bm, Cm, workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))
    whole = torch.empty(-(-need // 4), device="cuda")
    assert torch.equal(bp.ssm_scan(u, dt, A, Bm, Cm, workspace=whole), bp.ssm_scan(u, dt, A, Bm, Cm))
    states = torch.empty(bp.ssm_scan_states(T, 1, D, N).numel() + 8, dtype=torch.uint8, device="cuda")
    with pytest.raises(bp.BppsaError):
        bp.ssm_scan(u, dt, A, Bm, Cm, states=states[8:])


def test_new_arrays_have_their_channels_side_by_side():
    import torch
    from paper_1907_10134_amd.ssm import _like
    x = torch.empty(1000)
    for shape, strides in (((12, 3, 20), (1, 40, 1)), ((12, 3, 20), (40, 1, 1)), ((12, 3, 20), (0, 20, 1)), ((12, 3, 20), (20, 0, 1)),
                           ((12, 3, 20), (0, 0, 1)), ((12, 20), (1, 1)), ((12, 3, 20), (20, 300, 1)), ((1, 3, 20), (1, 20, 1))):
        new = _like(x.as_strided(shape, strides))
        assert new.shape == shape and new.stride(-1) == 1 and new.numel() == len({i for i in _offsets(new)}), strides


def _offsets(x):
    import itertools
    return (sum(i * s for i, s in zip(at, x.stride())) for at in itertools.product(*map(range, x.shape)))
