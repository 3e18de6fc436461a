"""GPU: the state space layer's operators together, as a small model that is trained and served."""
import pytest

pytestmark = pytest.mark.gpu


def test_training_brings_the_loss_down_and_is_the_same_every_time():
    import torch
    from workloads.ssm_stack import SsmStack, delayed
    losses = []
    for _ in range(2):
        stack = SsmStack(layers=2, width=64)
        run = []
        for step in range(60):
            s = delayed(48, 16, seed=step).cuda()
            run.append(stack.train_step(s[:-1], s[1:]))
        losses.append(torch.stack(run))
    first, last = float(losses[0][:5].mean()), float(losses[0][-5:].mean())
    assert torch.equal(losses[0], losses[1]) or float((losses[0] - losses[1]).abs().max()) < 0.05 * first     # the products are torch's
    assert last < 0.7 * first, (first, last)


def test_gradients_of_the_whole_step_against_differences():
    """The step's gradient along its own direction: bfloat16 activations of a stack of two layers round each term of the loss
    to 2^-9, so a difference over a change of some percent of the loss is good to some percent of it."""
    import torch
    from workloads.ssm_stack import SsmStack, delayed
    stack = SsmStack(layers=2, width=32, state_bits=32, lr=0.0)
    s = delayed(33, 8, seed=3).cuda()
    lengths = torch.tensor([33, 20, 1, 7, 33, 12, 30, 2], dtype=torch.int32, device="cuda")
    loss = lambda: float(stack.train_step(s[:-1], s[1:], lengths))
    loss()
    grads = {k: v.clone() for k, v in stack.g.items()}
    size = float(sum(v.square().sum() for v in grads.values())) ** 0.5

    def at(step):
        for k, v in stack.p.items():
            v.add_(grads[k], alpha=step / size)
            stack.w[k].copy_(v)
        return loss()

    eps = 0.05
    up = at(eps)
    down = at(-2 * eps)
    at(eps)
    assert abs((up - down) / (2 * eps) - size) < 0.1 * size, ((up - down) / (2 * eps), size)


def test_a_prompt_and_its_tokens_are_the_whole_sequence():
    """Ragged prompts, then tokens of the streams in slots of a larger cache, one row unused: the logits of the sequence at
    once, to bfloat16's rounding of the stream (2^-8 of values of some units, two layers)."""
    import torch
    from workloads.ssm_stack import SsmStack, delayed
    stack = SsmStack(layers=2, width=64)
    s = delayed(30, 3, seed=5).cuda()
    whole = stack.forward(s[:-1])
    lengths = torch.tensor([11, 1, 20], dtype=torch.int32, device="cuda")
    caches, cache = stack.caches(3), stack.caches(8)
    first = stack.forward(s[:20], lengths, caches=caches)
    slots = torch.tensor([6, -1, 0, 3], dtype=torch.int32, device="cuda")      # of streams 0, none, 1, 2
    of = [0, 0, 1, 2]
    for (h, last), (all_h, all_last) in zip(caches, cache):
        for row, stream in ((0, 0), (2, 1), (3, 2)):
            all_h[slots[row]], all_last[slots[row]] = h[stream], last[stream]
    for stream in range(3):
        n = int(lengths[stream])
        assert float((first[n - 1, stream] - whole[n - 1, stream]).abs().max()) < 0.15
    for k in range(8):
        tokens = torch.stack([s[int(lengths[b]) + k, b] for b in of])
        logits = stack.token(tokens, cache, slots)
        for row, stream in ((0, 0), (2, 1), (3, 2)):
            at = int(lengths[stream]) + k
            assert float((logits[row] - whole[at, stream]).abs().max()) < 0.15, (k, stream)
