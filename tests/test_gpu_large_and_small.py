"""GPU: the gated recurrence, the loss against top logits and the beam search at the ends of the sizes that they take."""
import numpy as np
import pytest

from oracle import gated
from test_gpu_beam import _case as _beams
from test_gpu_beam import _check as _check_beams
from test_gpu_distil import TYPES, _case, _check
from test_gpu_gated import _case as _layer
from test_gpu_gated import _close, _f32, _f64

pytestmark = pytest.mark.gpu


def test_more_tiles_in_a_row_than_run_at_once():
    """One chain of 782 tiles forward and 1563 backward, where some 512 workgroups run at a time."""
    import torch
    import paper_1907_10134_amd as bp
    T, B, D = 100000, 1, 3
    c, ref, dy, dy_ref, dh_last = _layer(51, T, B, D, "bfloat16", True, True, False, "tb")
    states, last, dh0 = bp.gated_scan_states(T, B, D), torch.empty((B, D), device="cuda"), torch.empty((B, D), device="cuda")
    y_ref, last_ref, _ = gated.scan(**ref)
    _close(bp.gated_scan(**c, states=states, h_last=last), y_ref, "bfloat16", "y")
    _close(last, last_ref, "float32", "h_last")
    g = bp.gated_scan_backward(dy, states=states, dh_last=dh_last, dh0=dh0, **c)
    want = gated.scan_backward(dy_ref, **ref, dh_last=_f64(dh_last))
    for name in ("dx", "dr", "di", "dz"):
        _close(getattr(g, name), want[name], "bfloat16", name)
    _close(dh0, want["dh0"], "float32", "dh0")
    again = bp.gated_scan_backward(dy, states=states, dh_last=dh_last, dh0=dh0, **c)
    assert all(torch.equal(a, b) for a, b in zip(g[:7], again[:7]))


@pytest.mark.parametrize("dtype", ("float16", "float32"))
def test_as_many_channels_as_there_may_be(dtype):
    import torch
    import paper_1907_10134_amd as bp
    T, B, D = 2, 1, 1 << 24
    rng = np.random.default_rng(52)
    put = lambda scale=1.0: torch.from_numpy((scale * rng.standard_normal((T, B, D), dtype=np.float32))).to(getattr(torch, dtype)).cuda()
    x, r, i, decay, h0 = put(), put(0.5), put(0.5), _f32(rng.uniform(0.04, 2.0, D)), _f32(rng.standard_normal((B, D)))
    states = bp.gated_scan_states(T, B, D)
    y = bp.gated_scan(x, r, i, decay, h0=h0, states=states)
    ref = dict(x=_f64(x), r=_f64(r), i=_f64(i), decay=_f64(decay), h0=_f64(h0))
    _close(y, gated.scan(**ref)[0], dtype, "y")
    g = bp.gated_scan_backward(y, x, r, i, decay, states, h0=h0)
    want = gated.scan_backward(_f64(y), **ref)
    _close(g.dx, want["dx"], dtype, "dx")
    _close(g.ddecay, want["ddecay"], "float32", "ddecay", sums=64)
    state = h0.clone()
    _close(bp.gated_scan_step(x[0], r[0], i[0], decay, state), gated.scan(**ref)[0][0], dtype, "a token's y")
    with pytest.raises(bp.BppsaError):
        bp.gated_scan(*(torch.zeros((1, 1, D + 1), dtype=x.dtype, device="cuda") for _ in range(3)), torch.ones(D + 1, device="cuda"))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", (1, 2, 16, 100))
def test_more_entries_than_tokens(V, dtype):
    """256 entries of a small vocabulary, each token many times over."""
    import paper_1907_10134_amd as bp
    import torch
    rng = np.random.default_rng(V)
    R, K = 5, 256
    c, ref = _case(53, R, V, 1, dtype, False, 0.3, False, 1.0)
    index, top = rng.integers(0, V, (R, K)), rng.standard_normal((R, K)).astype(np.float32)
    c["top_index"], c["top_logits"] = torch.from_numpy(index.astype(np.int32)).cuda().view(R, 1, K), _f32(top).view(R, 1, K)
    ref["top_index"], ref["top_logits"] = index, top.astype(np.float64)
    _check(bp.distil(**c), c, ref, dtype)


def test_as_many_rows_as_there_may_be():
    """The same few rows over and over, 2^22 - 1 of them, and one more, which is refused."""
    import torch
    import paper_1907_10134_amd as bp
    c, ref = _case(54, 7, 5, 2, "bfloat16", True, 0.3, False, 2.0)
    want = bp.distil(**c)
    _check(want, c, ref, "bfloat16")
    n = (1 << 22) - 1
    at = torch.arange(n, device="cuda") % 7
    many = {k: v[at].contiguous() if isinstance(v, torch.Tensor) else v for k, v in c.items()}
    got = bp.distil(**many)
    assert torch.equal(got.loss, want.loss[at]) and torch.equal(got.dlogits, want.dlogits[at])
    with pytest.raises(bp.BppsaError):
        bp.distil(**{k: torch.cat((v, v[:1])) if isinstance(v, torch.Tensor) else v for k, v in many.items()})


@pytest.mark.parametrize("size", [(1, 32, 524288), (3, 32, 131072), (700, 32, 33), (5000, 1, 40)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", TYPES)
def test_many_beams_of_large_vocabularies(size, dtype):
    import paper_1907_10134_amd as bp
    c = _beams(sum(size), *size, dtype)
    _check_beams(bp.beam_select(**c), c)


def test_states_of_one_slot_and_of_many_pieces():
    """One byte a slot, and a slot of 2^20 pieces and a bit."""
    import torch
    import paper_1907_10134_amd as bp
    n = (1 << 34) + 3
    big, small = torch.zeros((2, n), dtype=torch.uint8, device="cuda"), torch.zeros((2, 1), dtype=torch.uint8, device="cuda")
    big[0, ::4097], big[0, -1], small[0] = 7, 9, 3
    at = torch.zeros(1, dtype=torch.int32, device="cuda")
    bp.BeamStates([big, small]).move(at, at + 1)
    assert torch.equal(big[0], big[1]) and int(small[1]) == 3
