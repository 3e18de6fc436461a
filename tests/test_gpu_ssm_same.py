"""GPU: a training run of the small stack twice, bit by bit, with torch's own operations held to fixed orders of their sums."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("state_bits", (8, 32))
def test_a_training_run_has_the_same_bits_every_time(state_bits):
    """Losses, gradients, parameters and moments of two runs.  (torch also fills new memory with NaN in this mode: nothing may be
    read of an array before it is written.)"""
    import torch
    from workloads.ssm_stack import SsmStack, delayed
    was, warn = torch.are_deterministic_algorithms_enabled(), torch.is_deterministic_algorithms_warn_only_enabled()
    torch.use_deterministic_algorithms(True)
    try:
        runs = []
        for _ in range(2):
            stack = SsmStack(layers=2, width=64, state_bits=state_bits)
            lengths = torch.randint(1, 49, (16,), generator=torch.Generator().manual_seed(1)).to(torch.int32).cuda()
            losses = []
            for step in range(20):
                s = delayed(48, 16, seed=step).cuda()
                losses.append(stack.train_step(s[:-1], s[1:], lengths if step % 2 else None))
            runs.append((torch.stack(losses), stack))
        (a, first), (b, second) = runs
        assert bool(torch.isfinite(a).all()) and torch.equal(a, b)
        for name in ("p", "g", "w"):
            for k, v in getattr(first, name).items():
                assert torch.equal(v, getattr(second, name)[k]), (name, k)
        for name, held in first.optimiser.state.items():
            assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(held, second.optimiser.state[name])), name
    finally:
        torch.use_deterministic_algorithms(was, warn_only=warn)
