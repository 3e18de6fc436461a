"""GPU: the gated recurrence with as many columns and samples as are dealt out to the compute dies' own queues (64 and more), against
the fp64 oracle, and its calls on two streams."""
import pytest

from test_gpu_gated import TYPES, _case
from test_gpu_gated import test_scan_and_gradients as _scan_and_gradients

pytestmark = pytest.mark.gpu

# 63, 64, 65, 71 and 100 samples of one column; 13 and 20 samples of 5 and 10 columns in float32, of 3 and 5 in 16 bits; 129 of 2 and 1
SIZES = [(140, 63, 8), (140, 64, 3), (200, 65, 8), (300, 71, 5), (129, 100, 2), (200, 13, 300), (400, 20, 600), (257, 129, 65), (65, 130, 20)]


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gate,given,ragged,order", [(True, True, False, "tb"), (False, True, True, "bt")])
def test_many_chains(size, dtype, gate, given, ragged, order):
    _scan_and_gradients(size, dtype, gate, given, ragged, order)


@pytest.mark.parametrize("B", (1, 70))
def test_backward_passes_on_two_streams(B):
    """Side by side, each with a workspace of its own: the bits of a call by itself."""
    import torch
    import paper_1907_10134_amd as bp
    T, D = 2500, 130
    c, _, dy, _, dh_last = _case(43, T, B, D, "bfloat16", True, True, B > 1, "tb")
    states = bp.gated_scan_states(T, B, D)
    bp.gated_scan(**c, states=states)
    call = lambda stream=None: bp.gated_scan_backward(dy, states=states, dh_last=dh_last, stream=stream, **c)
    want = call()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[call(s) for s in streams] for _ in range(4)]
    torch.cuda.synchronize()
    for g in (g for pair in got for g in pair):
        assert all(torch.equal(a, b) for a, b in zip(g, want) if a is not None)
