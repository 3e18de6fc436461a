"""GPU: a beam search's step against the fp64 oracle."""
import numpy as np
import pytest

from oracle import beam

pytestmark = pytest.mark.gpu

TYPES = ("float32", "bfloat16", "float16")


def _f64(x):
    return x.detach().double().cpu().numpy()


def _case(seed, B, W, V, dtype, finished=True, first=True):
    import torch
    rng = np.random.default_rng(seed)
    c = {"logits": torch.from_numpy(2.5 * rng.standard_normal((B, W, V))).to(getattr(torch, dtype)).cuda()}
    scores = -np.sort(rng.uniform(0.0, 3.0, (B, W)), 1)
    if first and B > 1:
        scores[1, 1:] = -np.inf
    c["scores"] = torch.from_numpy(scores.astype(np.float32)).cuda()
    if finished:
        c["finished"], c["end"] = torch.from_numpy(rng.random((B, W)) < 0.3).cuda(), int(rng.integers(0, V))
    c["slots"] = torch.from_numpy(rng.permutation(B * W + 3)[:B * W].reshape(B, W).astype(np.int32)).cuda()
    return c


def _check(got, c):
    """Whole values are the oracle's; a score is its sum rounded once, 2^-24, and the logarithm of the sum is good to 2^-22."""
    ref = {k: v if isinstance(v, int) else v.cpu().numpy() if k in ("finished", "slots") else _f64(v) for k, v in c.items()}
    want = beam.select(**ref)
    for name, a, b in zip(got._fields[1:], got[1:], want[1:]):
        assert (a is None) == (b is None), name
        if a is not None:
            a = a.cpu().numpy()
            assert np.array_equal(a, b), (name, a[(a != b).any(-1)][:2], b[(a != b).any(-1)][:2])
    scores = _f64(got.scores)
    fine = np.isfinite(want[0])
    assert np.array_equal(fine, np.isfinite(scores)) and np.all(scores[~fine] == -np.inf)
    assert np.max(np.abs(scores[fine] - want[0][fine]) - 2.0 ** -22 - 2.0 ** -24 * np.abs(want[0][fine]), initial=0.0) <= 0
    return want


SIZES = [(1, 1, 1), (2, 3, 1), (1, 5, 3), (2, 4, 16), (3, 32, 7), (2, 32, 100), (3, 1, 8191), (2, 2, 8192), (2, 7, 8193), (1, 16, 20000), (5, 8, 4001),
         (2, 32, 50000), (1, 4, 131072), (1, 3, 524288), (40, 4, 300), (1, 31, 140001)]


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("finished", (False, True))
def test_selection(size, dtype, finished):
    import torch
    import paper_1907_10134_amd as bp
    c = _case(sum(size), *size, dtype, finished)
    got = bp.beam_select(**c)
    _check(got, c)
    again = bp.beam_select(**c)
    assert all(torch.equal(a, b) for a, b in zip(got, again) if a is not None)
    del c["slots"]
    less = bp.beam_select(**c)
    assert less.slots is less.sources is None and torch.equal(less.tokens, got.tokens) and torch.equal(less.scores, got.scores)


@pytest.mark.parametrize("V", (50, 700, 9000, 100000))
@pytest.mark.parametrize("W", (1, 4, 20))
def test_equal_logits(V, W):
    """All alike, alike but for one, of two values, zeros of both signs: the lowest tokens, many more than the bound leaves out."""
    import torch
    import paper_1907_10134_amd as bp
    B = 5
    x = torch.zeros((B, W, V), device="cuda")
    x[1, :, V // 2] = 1.0
    x[2] = torch.where(torch.arange(V, device="cuda") % 3 == 1, 0.5, -0.5)
    x[3] = torch.where(torch.arange(V, device="cuda") % 2 == 1, 0.0, -0.0)
    x[4, :, 2:] = float("-inf")
    scores = torch.zeros((B, W), device="cuda")
    scores[0, 1:] = float("-inf")
    for t in (torch.float32, torch.bfloat16):
        c = dict(logits=x.to(t), scores=scores)
        got = bp.beam_select(**c)
        _check(got, c)


def test_beams_alike_come_in_their_order():
    """The same logits and scores in every beam: sums that are equal to the last bit, in every size of a batch."""
    import torch
    import paper_1907_10134_amd as bp
    x = torch.randn((1, 1, 30000), device="cuda").expand(3, 6, 30000).contiguous()
    got = bp.beam_select(x, torch.zeros((3, 6), device="cuda"))
    best = x[0, 0].topk(1).indices
    assert bool((got.parents == torch.arange(6, device="cuda")).all()) and bool((got.tokens == best).all())


def test_masked_broken_and_dead_beams():
    """Rows of minus infinity, NaN and plus infinity count as minus infinity, scores that are not finite too; their logits do not
    reach other beams, and those of finished beams are not read."""
    import torch
    import paper_1907_10134_amd as bp
    inf, nan = float("inf"), float("nan")
    c = _case(3, 6, 4, 10000, "float32", finished=False, first=False)
    x = c["logits"]
    x[0, 0] = -inf
    x[1, 1, 77], x[2, 2, 9999] = nan, inf
    x[3, :, 5:] = -inf
    x[4] = nan
    c["scores"][0, 1], c["scores"][0, 2], c["scores"][0, 3] = nan, inf, -inf
    c["finished"], c["end"] = torch.zeros((6, 4), dtype=torch.bool, device="cuda"), 4
    c["finished"][4, 1] = c["finished"][1, 3] = True
    x[1, 3] = nan
    want = _check(bp.beam_select(**c), c)
    assert np.all(want[0][0] == -np.inf) and want[0][4, 0] == float(c["scores"][4, 1]) and np.all(want[0][4, 1:] == -np.inf)


@pytest.mark.parametrize("W", (1, 5, 32))
def test_vocabularies_with_few_tokens_left(W):
    """All but a few tokens masked with minus infinity, in one piece of a row or over several, fewer of them than beams; a NaN among
    masked tokens still breaks its row."""
    import torch
    import paper_1907_10134_amd as bp
    rng = np.random.default_rng(W)
    x = torch.full((6, W, 30000), float("-inf"), device="cuda")
    for b, places in enumerate(([29999], [0, 8191, 8192], range(100, 140), rng.integers(0, 30000, 300), [5, 9000, 17000, 25000], [7])):
        for w in range(W):
            for v in places:
                x[b, w, int(v)] = float(rng.standard_normal())
    x[4, 0, 20000] = float("nan")              # its piece has a finite token too
    x[5, W - 1, 12345] = float("nan")          # its piece has none
    for t in (torch.float32, torch.float16):
        c = dict(logits=x.to(t), scores=torch.zeros((6, W), device="cuda"))
        _check(bp.beam_select(**c), c)


def test_strides():
    """Beams first in memory, windows of wider rows, an odd offset."""
    import torch
    import paper_1907_10134_amd as bp
    for dtype in TYPES:
        c = _case(5, 3, 4, 9001, dtype)
        wide = torch.full((4, 3, 9010), float("nan"), dtype=c["logits"].dtype, device="cuda")
        wide[:, :, 3:9004] = c["logits"].transpose(0, 1)
        c["logits"] = wide.transpose(0, 1)[:, :, 3:9004]
        _check(bp.beam_select(**c), c)
        c["logits"] = c["logits"][:1, :1].expand(3, 4, 9001)
        _check(bp.beam_select(**c), c)


def test_rows_further_apart_than_32_bits_count():
    import torch
    import paper_1907_10134_amd as bp
    c = _case(6, 3, 3, 500, "bfloat16")
    wide = torch.empty((3, 3, 1 << 28), dtype=torch.bfloat16, device="cuda")
    wide[:, :, 7:507] = c["logits"]
    c["logits"] = wide[:, :, 7:507]
    _check(bp.beam_select(**c), c)


def test_states_move_to_the_children():
    """States of several types and sizes, of odd bytes too: the children's are their parents', all other slots as they were."""
    import torch
    import paper_1907_10134_amd as bp
    B, W, V = 5, 6, 40
    c = _case(7, B, W, V, "float32", finished=True)
    slots = int(c["slots"].max()) + 2
    tensors = [torch.randn((slots, 70, 16), device="cuda"), torch.randn((slots, 3, 70), device="cuda").to(torch.bfloat16),
               torch.randn((slots, 33), device="cuda"), torch.randint(0, 100, (slots, 9), device="cuda", dtype=torch.int32),
               torch.randint(0, 100, (slots, 7), device="cuda", dtype=torch.uint8), torch.randn((slots, 5000), device="cuda"),
               torch.randn(slots, device="cuda"), torch.randint(0, 2, (slots, 3, 16385), device="cuda", dtype=torch.bool)]
    before = [x.clone() for x in tensors]
    got = bp.beam_select(**c)
    states = bp.BeamStates(tensors)
    states.move(got.sources, got.slots)
    want = _check(got, c)
    old = c["slots"].cpu().numpy()
    for x, was in zip(tensors, before):
        left = set(range(slots))
        for b in range(B):
            for w in range(W):
                to, of = int(want[4][b, w]), int(old[b, want[1][b, w]])
                assert torch.equal(x[to], was[of]), (b, w)
                left.discard(to)
        for k in left:
            assert torch.equal(x[k], was[k])
    # rows of no stream, and one that stays where it is
    now = [x.clone() for x in tensors]
    states.move(torch.tensor([-1, slots, 0, 2], dtype=torch.int32, device="cuda"), torch.tensor([0, 1, -1, 2], dtype=torch.int32, device="cuda"))
    assert all(torch.equal(a, b) for a, b in zip(tensors, now))


def test_more_rows_than_a_launch_has():
    """5000 rows in slots of a large state, every other one copied to its neighbour."""
    import torch
    import paper_1907_10134_amd as bp
    n = 10000
    x, y = torch.randn((n, 300), device="cuda"), torch.arange(n, device="cuda", dtype=torch.int16).view(n, 1).contiguous()
    want = [x.view(n // 2, 2, 300)[:, :1].expand(-1, 2, -1).reshape(n, 300).clone(), (y // 2 * 2)]
    at = torch.arange(0, n, 2, device="cuda", dtype=torch.int32)
    bp.BeamStates([x, y]).move(at, at + 1)
    assert torch.equal(x, want[0]) and torch.equal(y, want[1])


def test_slots_further_apart_than_32_bits_count():
    import torch
    import paper_1907_10134_amd as bp
    x = torch.zeros((9, 1 << 29), dtype=torch.uint8, device="cuda")
    x[7] = 5
    bp.BeamStates([x]).move(torch.tensor([7], dtype=torch.int32, device="cuda"), torch.tensor([8], dtype=torch.int32, device="cuda"))
    assert bool((x[8] == 5).all()) and int(x[0, 0]) == 0 and int(x[6].max()) == 0


def test_another_stream_and_a_graph():
    import torch
    import paper_1907_10134_amd as bp
    c = _case(8, 4, 5, 20000, "bfloat16")
    slots = int(c["slots"].max()) + 1
    state = torch.randn((slots, 1000), device="cuda")
    first = state.clone()
    states = bp.BeamStates([state])

    def work(stream=None):
        got = bp.beam_select(stream=stream, **c)
        states.move(got.sources, got.slots, stream=stream)
        return got

    want = work()
    moved = state.clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    state.copy_(first)
    torch.cuda.synchronize()
    got = work(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(state, moved)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = work()
    for _ in range(3):
        for x in held:
            x.zero_()
        state.copy_(first)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want)) and torch.equal(state, moved)
        assert torch.equal(bp.beam_select(**c).tokens, want.tokens)


def test_two_streams_at_once():
    """Each call has a workspace of its own: two searches side by side are what they are by themselves."""
    import torch
    import paper_1907_10134_amd as bp
    torch.manual_seed(5)
    x = [torch.randn((9, 7, 30001), device="cuda").bfloat16() for _ in range(2)]
    s = torch.randn((9, 7), device="cuda")
    want = [bp.beam_select(y, s) for y in x]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[bp.beam_select(y, s, stream=q) for y, q in zip(x, streams)] for _ in range(4)]
    torch.cuda.synchronize()
    for pair in got:
        for a, b in zip(pair, want):
            assert torch.equal(a.scores, b.scores) and torch.equal(a.tokens, b.tokens) and torch.equal(a.parents, b.parents)


def test_refusals():
    import torch
    import paper_1907_10134_amd as bp
    c = _case(9, 2, 4, 60, "float32")
    bad = lambda **k: pytest.raises(ValueError, bp.beam_select, **dict(c, **k))
    bad(logits=c["logits"].double())
    bad(logits=c["logits"][0])
    bad(logits=c["logits"].cpu())
    bad(logits=c["logits"].transpose(1, 2).contiguous().transpose(1, 2))
    bad(scores=c["scores"].double())
    bad(scores=c["scores"][:1])
    bad(finished=c["finished"].int())
    bad(end=60)
    bad(end=-1)
    bad(slots=c["slots"].long())
    with pytest.raises(TypeError):
        bp.beam_select(c["logits"], None)
    with pytest.raises(bp.BppsaError):
        bp.beam_select(torch.zeros((1, 33, 50), device="cuda"), torch.zeros((1, 33), device="cuda"))
    with pytest.raises(bp.BppsaError):
        bp.beam_select(torch.zeros((1, 1, (1 << 19) + 1), device="cuda"), torch.zeros((1, 1), device="cuda"))
    x = torch.zeros((4, 6), device="cuda")
    for tensors in ([x[:, ::2]], [x, x[:3]], [x.cpu()], [x, torch.zeros((4, 0), device="cuda")]):
        with pytest.raises(ValueError):
            bp.BeamStates(tensors)
    s, i = bp.BeamStates([x]), torch.zeros(2, dtype=torch.int32, device="cuda")
    for pair in ((i.long(), i), (i, i.long()), (i[:1], i)):
        with pytest.raises(ValueError):
            s.move(*pair)
    with pytest.raises(TypeError):
        s.move(None, i)
