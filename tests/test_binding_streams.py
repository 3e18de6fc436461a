"""The dense, sparse and training calls of the binding on a stream of the caller's choice."""
import inspect

import pytest

CALLS = ("head_seed", "build_jacobians", "scan", "scan_h20_diag", "scan_h128_diag", "scan_h128_relay_diag", "rnn_scan_fused", "gru_scan_fused",
         "gru_scan_fused_relay_diag", "param_grads", "head_backward", "csr_conv3x3", "csr_conv2d", "csr_linear", "csr_relu",
         "csr_maxpool2x2", "spmv")


@pytest.mark.parametrize("name", CALLS)
def test_every_call_hands_all_its_arguments_over(monkeypatch, name):
    from paper_1907_10134_amd import binding
    call, got = getattr(binding, name), []
    monkeypatch.setattr(binding, "_aside", lambda stream, again, *args: got.append((stream, again, args)))
    names = list(inspect.signature(call).parameters)
    call(**dict({k: k for k in names}, stream="side"))
    want = [None if k == "stream" else k for k in names]
    assert got == [("side", call, tuple(want[:-1] if want[-1] is None else want))]


def test_no_call_that_makes_something_is_left_out():
    """Whatever takes a stream and makes an array or a workspace goes through _aside."""
    from paper_1907_10134_amd import binding
    for name, f in inspect.getmembers(binding, inspect.isfunction):
        if f.__module__ == binding.__name__ and "stream" in inspect.signature(f).parameters and not name.startswith("_"):
            text = inspect.getsource(f)
            if "torch.empty" in text or "_workspace(" in text or "_two_call(" in text:
                assert name in CALLS, name


@pytest.mark.gpu
def test_memory_of_results_on_another_stream_is_not_given_out_again():
    import torch
    import paper_1907_10134_amd as bp
    T, B, H, I = 200, 8, 20, 1
    r = lambda *shape: 0.2 * torch.randn(shape, device="cuda")
    h, x, w_ih, w_hh, b, seed = torch.tanh(r(T + 1, B, H)), r(T, B, I), r(H, I), r(H, H), r(H), r(B, H)
    conv, mask = r(4, 3, 3, 3), torch.ones((4, 3, 3, 3), dtype=torch.uint8, device="cuda")
    ones = torch.ones(4 * 8 * 8, device="cuda")

    def work(stream):
        Jt = bp.build_jacobians(bp.RNN_TANH, h, w_hh=w_hh, stream=stream)
        G = bp.scan(Jt, seed, stream=stream)
        fused = bp.rnn_scan_fused(h, w_hh, seed, stream=stream)
        A = bp.csr_conv3x3(conv, mask, 8, 8, stream=stream)
        return [Jt, G, fused, *bp.param_grads(bp.RNN_TANH, h, x, G, stream=stream), A.indptr, A.indices, A.data,
                bp.spmv(A, ones, stream=stream)]

    want = work(None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = work(side)
    sizes, places = [(x.shape, x.dtype) for x in got], {x.data_ptr() for x in got}
    kept = got[3]
    del got
    new = [torch.empty(shape, dtype=t, device="cuda") for shape, t in sizes for _ in range(2)]
    assert not places & {x.data_ptr() for x in new}
    side.synchronize()
    bp.check_scan()
    assert torch.equal(kept, want[3])
    side.wait_stream(torch.cuda.current_stream())
    got = work(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
