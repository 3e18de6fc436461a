"""CPU: how 8-bit first moments are held, as the oracle says it: a value that nothing feeds any more has to reach zero."""
import numpy as np
import pytest

from oracle import ssm


def _run(beta1, steps, held):
    """m of a block of 256 after 60 steps of gradients and `steps` more in which the last eight get none, in units of the scale."""
    rng, m, t = np.random.default_rng(1), np.zeros(256), 0
    for t in range(60 + steps):
        g = rng.standard_normal(256)
        if t >= 60:
            g[248:] = 0
        x = beta1 * m + (1 - beta1) * g
        scale = np.max(np.abs(x)) / 448
        m = held(x / scale, np.abs(x) < np.abs(m), beta1, ssm.chance_of_m(t, 0, 256)) * scale
    return m / scale


@pytest.mark.parametrize("beta1,steps", [(0.9, 600), (0.9375, 800), (0.95, 1200), (0.99, 4000)])
def test_a_first_moment_that_nothing_feeds_reaches_zero(beta1, steps):
    m = _run(beta1, steps, lambda *a: ssm.held_m(*a)[0])
    assert not np.any(m[248:]) and np.count_nonzero(m[:248]) > 200


def test_to_the_nearest_alone_it_would_not():
    """Why values go by chance: 4 spacings of 2^-9 are 3.6 a step later, and 4 again.  From 2^-6 on a beta1 of up to 15/16 moves every
    value of the grid, one of 0.95 does not move 9/16 of any size while the scale stays."""
    nearest = lambda q, shrinks, beta1, by: ssm.held_m(q, np.zeros_like(shrinks), 0.0, by)[0]
    assert np.all(np.abs(_run(0.9, 600, nearest)[248:]) >= 2.0 ** -9)
    normal = ssm.e4m3_values()[8:]
    kept = lambda beta1: nearest(beta1 * normal, normal > 0, 0.0, 0.0) >= normal
    assert not np.any(kept(0.9)) and not np.any(kept(15 / 16)[1:]) and np.count_nonzero(kept(0.95)) >= 14


def test_the_values_held_are_torchs_nearest_or_the_neighbours():
    import torch
    rng = np.random.default_rng(2)
    q = rng.standard_normal(4000) * np.exp(rng.uniform(-8, 6, 4000))
    q = q[np.abs(q) < 448].astype(np.float32).astype(np.float64)
    shrinks = rng.random(len(q)) < 0.5
    got, by_chance = ssm.held_m(q, shrinks, 0.9, rng.random(len(q)))
    nearest = torch.from_numpy(q).float().to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(got[~by_chance], nearest[~by_chance]) and np.any(got[by_chance] != nearest[by_chance])
    assert np.all(np.abs(got - q)[by_chance] < 2.0 ** -9) and np.all(by_chance == (shrinks & (np.abs(q) < 2.0 ** -6)))
