"""GPU: gated layers, the loss against a teacher's top logits and the beam search together, as a small stack that is trained and
served."""
import pytest

pytestmark = pytest.mark.gpu


def _top(stack, tokens, lengths=None, k=4):
    top, index = stack.forward(tokens, lengths).topk(k)
    return top.contiguous(), index.int()


def test_gradients_of_the_whole_step_against_differences():
    """The step's gradient along its own direction, as of the stack without these parts: bfloat16 activations of two layers round
    each term of the loss to 2^-9, so a difference over a change of some percent of the loss is good to some percent of it."""
    import torch
    from workloads.ssm_stack import SsmStack, delayed
    teacher = SsmStack(layers=2, width=64, seed=5)
    stack = SsmStack(layers=2, width=32, state_bits=32, lr=0.0, gated=(0,))
    s = delayed(33, 8, seed=3).cuda()
    lengths = torch.tensor([33, 20, 1, 7, 33, 12, 30, 2], dtype=torch.int32, device="cuda")
    top, index = _top(teacher, s[:-1], lengths)
    top = 4 * top                              # a teacher that is surer than random weights are: a loss of some size
    norm = torch.logsumexp(4 * teacher.forward(s[:-1], lengths), -1)
    for how in ({}, dict(top_norm=norm), dict(temperature=2.0, hard=0.5, targets=s[1:].int())):
        loss = lambda: float(stack.distil_step(s[:-1], top, index, lengths, **how))
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
        assert abs((up - down) / (2 * eps) - size) < 0.1 * size, (how.keys(), (up - down) / (2 * eps), size)
        assert float(stack.g["gate_proj0"].abs().max()) > 0 and float(stack.g["decay_log0"].abs().max()) > 0


def test_steps_run_and_give_finite_weights():
    import torch
    from workloads.ssm_stack import SsmStack, delayed
    teacher, stack = SsmStack(layers=2, width=64, seed=5), SsmStack(layers=3, width=32, gated=(0, 2))
    for step in range(8):
        s = delayed(48, 16, seed=step).cuda()
        loss = stack.distil_step(s[:-1], *_top(teacher, s[:-1])) if step % 2 else stack.train_step(s[:-1], s[1:])
        assert bool(torch.isfinite(loss))
    assert all(bool(torch.isfinite(v).all()) for v in stack.p.values())


def test_a_prompt_and_its_tokens_are_the_whole_sequence():
    """Ragged prompts, then tokens of the streams in slots of a larger cache, one row unused: the logits of the sequence at once, to
    bfloat16's rounding of the stream (2^-8 of values of some units, two layers)."""
    import torch
    from workloads.ssm_stack import SsmStack, delayed
    stack = SsmStack(layers=2, width=64, gated=(1,))
    s = delayed(30, 3, seed=5).cuda()
    whole = stack.forward(s[:-1])
    lengths = torch.tensor([11, 1, 20], dtype=torch.int32, device="cuda")
    caches, cache = stack.caches(3), stack.caches(8)
    stack.forward(s[:20], lengths, caches=caches)
    slots = torch.tensor([6, -1, 0, 3], dtype=torch.int32, device="cuda")      # of streams 0, none, 1, 2
    rows = ((0, 0), (2, 1), (3, 2))
    for have, all_ in zip(caches, cache):
        for a, b in zip(have, all_):
            for row, stream in rows:
                b[slots[row]] = a[stream]
    for k in range(8):
        tokens = torch.stack([s[int(lengths[b]) + k, b] for b in (0, 0, 1, 2)])
        logits = stack.token(tokens, cache, slots)
        for row, stream in rows:
            assert float((logits[row] - whole[int(lengths[stream]) + k, stream]).abs().max()) < 0.15, (k, stream)


def test_one_beam_is_the_greedy_continuation():
    import torch
    from workloads.ssm_stack import SsmStack, delayed
    stack = SsmStack(layers=2, width=64, gated=(0,))
    s = delayed(20, 4, seed=9).cuda()
    found, _ = stack.beams(s, 1, 12)
    caches = stack.caches(4)
    logits = stack.forward(s, caches=caches)[-1]
    for k in range(12):
        token = logits.argmax(-1)
        assert torch.equal(found[:, 0, k].long(), token), k
        logits = stack.token(token, caches)


def test_beams_are_what_a_search_without_caches_finds():
    """Every beam's score is the sum of the log shares that the whole sequence has: a logit is good to 0.15 there and here, a log
    share to twice that, as many times as there are steps.  The beams differ, and come best first."""
    import torch
    from workloads.ssm_stack import SsmStack, delayed
    stack = SsmStack(layers=2, width=64, gated=(1,))
    s = delayed(12, 3, seed=4).cuda()
    lengths = torch.tensor([13, 4, 1], dtype=torch.int32, device="cuda")
    width, steps, end = 5, 7, 3
    found, scores = stack.beams(s, width, steps, lengths=lengths, end=end)
    assert bool((scores[:, :-1] >= scores[:, 1:]).all())
    for b in range(3):
        rows = found[b].tolist()
        assert len(set(map(tuple, rows))) == width
        for w, row in enumerate(rows):
            n = row.index(end) + 1 if end in row else steps
            assert all(t == end for t in row[n:])
            prompt = s[:int(lengths[b]), b].tolist()
            tokens = torch.tensor(prompt + row[:n], device="cuda")[:, None]
            logp = torch.log_softmax(stack.forward(tokens[:-1])[len(prompt) - 1:, 0].double(), -1)
            want = float(sum(logp[k, row[k]] for k in range(n)))
            assert abs(float(scores[b, w]) - want) < 0.3 * n, (b, w, float(scores[b, w]), want)
