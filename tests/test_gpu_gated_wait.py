"""The wait between tiles of the gated recurrence: what it makes of words that are there, and that it ends where they are not."""
import ctypes

import numpy as np
import pytest

from test_oracle_ssm import EINVAL, ONE, lib  # noqa: F401

EMPTY, SETTLED = (1 << 64) - 1, 0x80000000 << 32


def _bits(x):
    return int(np.float32(x).view(np.uint32))


def _wait(words, looks):
    """The states of the 64 channels, as float32."""
    import torch
    from paper_1907_10134_amd import gated
    call = gated._lib.bppsa_gated_wait_diag
    call.restype, call.argtypes = ctypes.c_int, [ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p]
    w = torch.from_numpy(np.array(words, dtype=np.uint64).view(np.int64)).cuda()
    h = torch.full((64,), 7.0, device="cuda")
    assert call(w.data_ptr(), len(words), looks, h.data_ptr(), torch.cuda.current_stream().cuda_stream) == 0
    return h.cpu().numpy()


def _words(rng, tiles, settled):
    """Shares of all tiles and 64 channels; those of tile 0, and of settled[channel], the states themselves."""
    p, e = rng.uniform(0.1, 0.9, (tiles, 64)).astype(np.float32), rng.standard_normal((tiles, 64)).astype(np.float32)
    words = [[_bits(p[t, c]) << 32 | _bits(e[t, c]) for c in range(64)] for t in range(tiles)]
    want = np.zeros(64, dtype=np.float64)
    for c in range(64):
        for t in range(tiles):
            if t == 0 or t == settled[c]:
                words[t][c] = SETTLED | _bits(e[t, c])
                want[c] = e[t, c]
            else:
                want[c] = np.float64(p[t, c]) * want[c] + e[t, c]
    return words, want


@pytest.mark.gpu
@pytest.mark.parametrize("tiles", (1, 2, 3, 4, 5, 8, 9, 40, 1001))
def test_states_of_words_that_are_there(tiles):
    """From the nearest state over the shares behind it: products below 0.9 keep at most 10 roundings of 2^-24 of values below 40."""
    rng = np.random.default_rng(tiles)
    for settled in ([0] * 64, [tiles - 1] * 64, rng.integers(0, tiles, 64)):
        words, want = _words(rng, tiles, settled)
        assert np.max(np.abs(_wait(words, 1 << 12) - want)) <= 10 * 40 * 2.0 ** -24


@pytest.mark.gpu
@pytest.mark.parametrize("tiles,gone", [(1, 0), (3, 0), (3, 2), (9, 0), (9, 4), (9, 8), (40, 17)])
@pytest.mark.parametrize("looks", (1, 2, 50, 1000))
def test_a_wait_for_what_never_comes_ends(tiles, gone, looks):
    """A word of one channel is missing in front of every state that is known: that channel is NaN after so many looks, also where its
    later products are zero.  The wave goes together, so the others may be given up with it: they are right or NaN, never a number
    that is wrong."""
    rng = np.random.default_rng(tiles + gone)
    words, want = _words(rng, tiles, [0] * 64)
    words[gone][5] = EMPTY
    if gone + 1 < tiles:
        words[gone + 1][5] = _bits(0.0) << 32 | _bits(1.0)
    h = _wait(words, looks)
    assert np.isnan(h[5])
    others = np.delete(np.arange(64), 5)
    assert np.all(np.isnan(h[others]) | (np.abs(h[others] - want[others]) <= 10 * 40 * 2.0 ** -24))
    if tiles <= 4:                             # all in the one window that is looked at
        assert not np.any(np.isnan(h[others]))


@pytest.mark.gpu
def test_what_is_missing_behind_a_known_state_does_not_matter():
    rng = np.random.default_rng(3)
    words, want = _words(rng, 9, [6] * 64)
    for t in range(6):
        words[t] = [EMPTY] * 64
    assert np.max(np.abs(_wait(words, 4) - want)) <= 10 * 40 * 2.0 ** -24


def test_bad_arguments_are_rejected_before_any_launch(lib):  # noqa: F811
    one = ctypes.c_void_p(ONE)
    call = lambda w=one, tiles=2, looks=5, h=one: lib.bppsa_gated_wait_diag(w, tiles, looks, h, None)
    assert call(w=None) == call(w=ctypes.c_void_p(ONE + 4)) == call(tiles=0) == call(looks=0) == call(looks=(1 << 24) + 1) == call(h=None) == EINVAL
