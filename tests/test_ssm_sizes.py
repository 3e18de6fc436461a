"""CPU: sizes that no launch or no count of bytes can hold are refused before anything is launched."""
import ctypes

from test_oracle_ssm import EINVAL, EOVERFLOW, EWORKSPACE, ONE, Grads, Rows, _rows, _ssm, lib  # noqa: F401 (a fixture)

MOST = 0x7FFFFFFF


def _backward(lib, l):
    g = Grads(_rows(), _rows(), Rows(), ONE, ONE, ONE, None, None, None)
    return lib.bppsa_ssm_scan_backward(ctypes.byref(l), ctypes.byref(_rows()), ctypes.c_void_p(ONE), ctypes.byref(g), None,
                                       ctypes.c_size_t(0), None)


def test_more_parameters_than_the_joining_launch_can_hold(lib):  # noqa: F811
    # (64 states + 2) 2^24 sums, 64 to a workgroup of 256: 4.4e9 threads; the last D below 2^24 workgroups goes on to the workspace
    assert _backward(lib, _ssm(T=1, B=1, D=1 << 24, N=64)) == EOVERFLOW
    assert _backward(lib, _ssm(T=1, B=1, D=16 << 20, N=49)) == EOVERFLOW
    assert _backward(lib, _ssm(T=1, B=1, D=16 << 20, N=48)) == EWORKSPACE
    assert _backward(lib, _ssm(T=1, B=1, D=15 << 20, N=64)) == EWORKSPACE


def test_more_pieces_than_a_launch_can_hold(lib):  # noqa: F811
    one, d = ctypes.c_void_p(ONE), ctypes.c_double
    for pieces in (1 << 24, 1 << 33):
        assert lib.bppsa_adamw_step(1, one, ctypes.c_int64(pieces), one, 0, 32, 1, d(1e-3), d(0.9), d(0.999), d(1e-8),
                                    ctypes.c_uint32(0), None) == EOVERFLOW


def test_sizes_of_which_the_bytes_do_not_fit_have_none(lib):  # noqa: F811
    assert lib.bppsa_ssm_scan_states_bytes(MOST, MOST, MOST, 64) == 0
    assert lib.bppsa_ssm_scan_states_bytes(1 << 30, 1 << 15, 1 << 20, 16) == 0
    assert lib.bppsa_ssm_scan_workspace_bytes(MOST, MOST, MOST, 64, 1) == 0
    assert lib.bppsa_ssm_scan_backward_workspace_bytes(MOST, MOST, MOST, 64, MOST) == 0
    assert lib.bppsa_ssm_conv_backward_workspace_bytes(MOST, MOST, MOST, 4) == 0
    assert lib.bppsa_ssm_conv_backward_workspace_bytes(1 << 20, 64, 8192, 4) > 1 << 32
    assert lib.bppsa_ssm_scan_backward_workspace_bytes(1 << 18, 4, 8192, 16, 1) > 1 << 30


def test_an_eps_or_lr_that_fp32_does_not_hold(lib):  # noqa: F811
    """The update divides by root + eps: a value that has had no gradient yet would become 0 / 0."""
    one, d = ctypes.c_void_p(ONE), ctypes.c_double
    for lr, eps in ((1e-3, 1e-40), (1e-3, 1e-50), (1e-3, float("nan")), (1e-3, 1e39), (1e39, 1e-8), (float("inf"), 1e-8)):
        assert lib.bppsa_adamw_step(1, one, ctypes.c_int64(1), one, 0, 32, 1, d(lr), d(0.9), d(0.999), d(eps), ctypes.c_uint32(0),
                                    None) == EINVAL, (lr, eps)
