"""GPU: the loss against a teacher's top logits and its gradient against the fp64 oracle."""
import numpy as np
import pytest

from oracle import distil

pytestmark = pytest.mark.gpu

TYPES = ("float32", "bfloat16", "float16")


def _f64(x):
    return x.detach().double().cpu().numpy()


def _on(a, t):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).to(t).cuda()


def _case(seed, R, V, K, dtype, tail, hard, masked, temperature, top_type="float32", spread=2.0):
    """Keyword arguments on the GPU, [R, 1, ...], and the same for the oracle from the rounded values."""
    import torch
    rng = np.random.default_rng(seed)
    teacher = spread * rng.standard_normal((R, V))
    c = {"logits": _on(teacher + rng.standard_normal((R, V)), getattr(torch, dtype)).view(R, 1, V)}
    index = np.argsort(-teacher, axis=1)[:, :K].astype(np.int32)
    top = np.take_along_axis(teacher, index, 1)
    if K > 2:
        index[::3, K // 2:] = -1
        top[1::4, 0] = -np.inf
    if R > 4:
        index[4] = -1                          # a row without entries
    c["top_logits"], c["top_index"] = _on(top, getattr(torch, top_type)).view(R, 1, K), _on(index, torch.int32).view(R, 1, K)
    if tail:
        c["top_norm"] = _on(np.log(np.exp(teacher / temperature).sum(1)), torch.float32).view(R, 1)
    if hard:
        target = rng.integers(0, V, R)
        target[::5] = -1
        target[1::5] = index[1::5, -1]         # one that is an entry too, or none
        c["targets"] = _on(target, torch.int32).view(R, 1)
    if masked:
        weight = rng.uniform(0.5, 2.0, R)
        weight[2::3] = 0.0
        c["weight"] = _on(weight, torch.float32).view(R, 1)
    ref = {k: _f64(v)[:, 0] for k, v in c.items()}
    for k in ("top_index", "targets"):
        if k in ref:
            ref[k] = ref[k].astype(int)
    if masked:                                 # rows of weight zero are not read
        c["logits"][2::3] = float("nan")
    more = dict(temperature=temperature, hard=hard)
    return dict(c, **more), dict(ref, **more)


def _check(got, c, ref, dtype):
    """Exponentials are good to 2^-23, and to 16 of 2^-24 where the arguments of 16-bit logits are rounded; a sum to as many
    roundings as it has terms in a row, at most V / 256 and the joining ones: relative to the shares, which are 1 at most."""
    import torch
    t = getattr(torch, dtype)
    loss, grad = distil.loss(**ref)
    V, tau, hard = ref["logits"].shape[1], ref["temperature"], ref["hard"]
    w = ref.get("weight", np.ones(len(loss)))
    rel = (32 + V / 256) * 2.0 ** -24
    g = _f64(got.loss).reshape(-1)
    assert np.all(np.isfinite(g))
    off = np.abs(g - loss) - (2 * w * ((1 - hard) * tau ** 2 + hard) * rel + 2.0 ** -23 * np.abs(loss))
    assert np.max(off) <= 0, ("loss", np.argmax(off), g[np.argmax(off)], loss[np.argmax(off)])
    if got.dlogits is None:
        return
    g = _f64(got.dlogits).reshape(grad.shape)
    half = torch.finfo(t).eps / 2
    off = np.abs(g - grad) - (half * np.abs(grad) + half * torch.finfo(t).tiny + (2 * w * ((1 - hard) * tau + hard) * rel)[:, None])
    assert np.all(np.isfinite(g)) and np.max(off) <= 0, ("dlogits", np.unravel_index(np.argmax(off), off.shape), np.max(np.abs(g - grad)))
    if "weight" in ref:
        assert np.all(g[w == 0] == 0)


SIZES = [(1, 1, 1), (3, 2, 2), (7, 16, 8), (9, 63, 5), (6, 64, 64), (5, 65, 1), (12, 255, 256 - 1), (6, 512, 256), (5, 513, 50), (5, 1000, 31),
         (6, 4001, 50), (4, 8192, 64), (3, 8193, 64), (3, 32001, 128), (3, 65537, 40), (5, 131073, 256), (2, 300001, 33),
         (2, 1024, 6), (3, 2049, 9), (3, 2048, 9), (4, 16384, 20), (4, 16385, 20), (1, 1 << 20, 40)]


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tail,hard,masked,temperature", [(False, 0.0, False, 1.0), (True, 0.0, True, 2.0), (False, 0.3, True, 0.7),
                                                          (True, 0.4, False, 1.0), (False, 1.0, False, 2.0)])
def test_loss_and_gradient(size, dtype, tail, hard, masked, temperature):
    import torch
    import paper_1907_10134_amd as bp
    R, V, K = size
    c, ref = _case(sum(size), R, V, K, dtype, tail, hard, masked, temperature)
    got = bp.distil(**c)
    _check(got, c, ref, dtype)
    alone = bp.distil(gradient=False, **c)
    assert alone.dlogits is None and torch.equal(alone.loss, got.loss)
    again = bp.distil(**c)
    assert torch.equal(again.loss, got.loss) and torch.equal(again.dlogits, got.dlogits), "the same bits on every call"
    c["logits"] = c["logits"].clone()
    place = bp.distil(dlogits=c["logits"], **c)
    assert place.dlogits is c["logits"] and torch.equal(place.dlogits, got.dlogits) and torch.equal(place.loss, got.loss)


@pytest.mark.parametrize("top_type", TYPES)
def test_types_of_the_entries(top_type):
    import paper_1907_10134_amd as bp
    c, ref = _case(3, 6, 777, 20, "bfloat16", True, 0.0, False, 1.0, top_type=top_type)
    _check(bp.distil(**c), c, ref, "bfloat16")


@pytest.mark.parametrize("V", (100, 5000, 140001))
def test_an_index_that_comes_twice_and_one_outside(V):
    """Shares of one token add up; what lies outside the vocabulary does not count, nor a target there."""
    import torch
    import paper_1907_10134_amd as bp
    c, ref = _case(4, 3, V, 6, "float32", False, 0.5, False, 1.0)
    for x, to in ((c["top_index"], lambda v: v), (ref["top_index"], lambda v: v)):
        x[1, ..., 2] = x[1, ..., 3]
        x[1, ..., 4] = V
        x[2, ..., 0] = -7
    for x in (c["targets"], ref["targets"]):
        x[2] = V
    _check(bp.distil(**c), c, ref, "float32")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", (40, 9001, 140001))
def test_rows_with_strides(dtype, V):
    """Sequence by sequence in memory, an odd row length inside a wider one: nothing beside the rows is written."""
    import torch
    import paper_1907_10134_amd as bp
    c, ref = _case(5, 6, V, 9, dtype, True, 0.0, True, 1.0)
    x = c["logits"].view(3, 2, V)
    wide = torch.full((2, 3, V + 5), 7.0, dtype=x.dtype, device="cuda")
    out = torch.full((2, 3, V + 3), 7.0, dtype=x.dtype, device="cuda")
    wide[:, :, 1:V + 1] = x.transpose(0, 1)
    more = {k: v.view(3, 2, *v.shape[2:]) if hasattr(v, "view") and k != "logits" else v for k, v in c.items()}
    more["logits"] = wide.transpose(0, 1)[:, :, 1:V + 1]
    got = bp.distil(dlogits=out.transpose(0, 1)[:, :, 2:V + 2], **more)
    _check(got, c, ref, dtype)
    assert bool((out[:, :, :2] == 7).all()) and bool((out[:, :, V + 2:] == 7).all())


def test_rows_without_the_dimension_of_the_samples():
    import torch
    import paper_1907_10134_amd as bp
    c, _ = _case(6, 5, 300, 7, "float32", True, 0.2, True, 1.0)
    want = bp.distil(**c)
    got = bp.distil(**{k: v.squeeze(1) if hasattr(v, "squeeze") else v for k, v in c.items()})
    assert got.loss.shape == (5,) and torch.equal(got.loss, want.loss[:, 0]) and torch.equal(got.dlogits, want.dlogits[:, 0])


@pytest.mark.parametrize("V", (30, 3000, 140001))
def test_logits_far_apart_and_tokens_that_are_masked(V):
    """Logits of the type's lowest and largest values and of minus infinity: finite losses where the entries have a share."""
    import torch
    import paper_1907_10134_amd as bp
    for dtype in TYPES:
        c, ref = _case(7, 4, V, 5, dtype, True, 0.0, False, 1.0)
        lowest = torch.finfo(getattr(torch, dtype)).min
        keep = set(ref["top_index"].flatten().tolist())
        others = [v for v in range(V) if v not in keep]
        for x in (c["logits"], ref["logits"]):
            x[0, ..., others[0]] = -np.inf
            x[1, ..., others[1]] = lowest
            x[2, ..., others[:-2]] = -np.inf
        _check(bp.distil(**c), c, ref, dtype)
        c["logits"][0, 0, others[2]] = float("nan")       # stays in its row
        got = bp.distil(**c)
        assert bool(torch.isnan(got.loss[0]).all()) and not bool(torch.isnan(got.loss[1:]).any())
        assert not bool(torch.isnan(got.dlogits[1:]).any())


def test_a_student_like_its_teacher():
    """Entries for the whole vocabulary with the student's own logits: no loss, no gradient."""
    import torch
    import paper_1907_10134_amd as bp
    x = torch.randn((5, 1, 200), device="cuda")
    index = torch.arange(200, device="cuda", dtype=torch.int32).expand(5, 1, 200).contiguous()
    got = bp.distil(x, x, index)
    assert float(got.loss.abs().max()) < 33 * 2.0 ** -24 and float(got.dlogits.abs().max()) < 33 * 2.0 ** -24


def test_gradient_against_differences():
    """Central differences of the kernel's own loss in float32, 2^-20 good, over 2e-2: 1e-4, and the third derivative's 1e-5."""
    import torch
    import paper_1907_10134_amd as bp
    c, ref = _case(8, 2, 60, 10, "float32", True, 0.3, False, 1.0)
    g = bp.distil(**c).dlogits
    for at in ((0, 0, int(ref["top_index"][0, 0])), (0, 0, 17), (1, 0, int(ref["targets"][1])), (1, 0, 3)):
        was = float(c["logits"][at])
        sums = []
        for d in (1e-2, -1e-2):
            c["logits"][at] = was + d
            sums.append(float(bp.distil(gradient=False, **c).loss.double().sum()))
        c["logits"][at] = was
        assert abs((sums[0] - sums[1]) / 2e-2 - float(g[at])) < 3e-4, at


def test_rows_further_apart_than_32_bits_count():
    import torch
    import paper_1907_10134_amd as bp
    c, ref = _case(9, 9, 64, 4, "bfloat16", False, 0.0, False, 1.0)
    wide = torch.empty((9, 1, 1 << 28), dtype=torch.bfloat16, device="cuda")
    wide[:, :, 8:72] = c["logits"]
    c["logits"] = wide[:, :, 8:72]
    _check(bp.distil(dlogits=wide[:, :, 100:164], **c), c, ref, "bfloat16")


def test_another_stream_and_a_graph():
    import torch
    import paper_1907_10134_amd as bp
    c, _ = _case(10, 40, 5000, 30, "bfloat16", True, 0.3, True, 2.0)
    want = bp.distil(**c)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = bp.distil(stream=side, **c)
    side.synchronize()
    assert torch.equal(got.loss, want.loss) and torch.equal(got.dlogits, want.dlogits)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = bp.distil(**c)
    for _ in range(3):
        held.loss.zero_(), held.dlogits.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(held.loss, want.loss) and torch.equal(held.dlogits, want.dlogits)
        assert torch.equal(bp.distil(**c).dlogits, want.dlogits)


def test_many_rows_and_two_streams():
    """More rows than 16 bits count, on two streams side by side: no call knows of the other."""
    import torch
    import paper_1907_10134_amd as bp
    c, ref = _case(12, 70001, 9, 3, "bfloat16", True, 0.3, True, 2.0)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[bp.distil(stream=s, **c) for s in streams] for _ in range(3)]
    torch.cuda.synchronize()
    _check(got[0][0], c, ref, "bfloat16")
    assert all(torch.equal(x.loss, got[0][0].loss) and torch.equal(x.dlogits, got[0][0].dlogits) for pair in got for x in pair)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", (7, 8, 9, 2047, 4095, 4096, 4097, 8191, 16383, 32769, 65535))
def test_rows_around_what_waves_hold(V, dtype):
    """As many entries as there may be, some of them twice, where rows begin to take more waves or chunks; every logit an odd
    number of elements off a multiple of 16 bytes."""
    import torch
    import paper_1907_10134_amd as bp
    K = min(V, 256)
    c, ref = _case(13, 3, V, K, dtype, True, 0.25, False, 1.5)
    if K > 4:
        for x in (c["top_index"], ref["top_index"]):
            x[1, ..., 1] = x[1, ..., 3]
    wide = torch.full((3, 1, V + 9), 3.0, dtype=c["logits"].dtype, device="cuda")
    wide[:, :, 1:V + 1] = c["logits"]
    c["logits"] = wide[:, :, 1:V + 1]
    got = bp.distil(**c)
    _check(got, c, ref, dtype)
    place = bp.distil(dlogits=c["logits"], **c)
    assert torch.equal(place.dlogits, got.dlogits) and torch.equal(place.loss, got.loss)
    assert bool((wide[:, :, 0] == 3).all()) and bool((wide[:, :, V + 1:] == 3).all())


def test_refusals():
    import torch
    import paper_1907_10134_amd as bp
    c, _ = _case(11, 4, 30, 5, "float32", True, 0.5, True, 1.0)
    bad = lambda **k: pytest.raises(ValueError, bp.distil, **dict(c, **k))
    bad(logits=c["logits"].double())
    bad(logits=c["logits"].cpu())
    bad(logits=c["logits"].transpose(1, 2).contiguous().transpose(1, 2)[..., ::2])
    bad(top_index=c["top_index"].long())
    bad(top_index=c["top_index"][..., :3])
    bad(top_logits=c["top_logits"][:2])
    bad(weight=c["weight"].half())
    bad(targets=c["targets"].long())
    bad(targets=None)
    bad(top_norm=c["top_norm"][:2])
    bad(dlogits=c["logits"].half())
    bad(loss=torch.empty(3, device="cuda"))
    for k in (dict(temperature=0.0), dict(temperature=float("nan")), dict(hard=1.5), dict(hard=-1.0)):
        with pytest.raises(bp.BppsaError):
            bp.distil(**dict(c, **k))
    with pytest.raises(bp.BppsaError):
        bp.distil(**dict(c, dlogits=torch.empty((1, 1, 30), device="cuda").expand(4, 1, 30)))
    big = torch.zeros((1, 1, 400), device="cuda")
    with pytest.raises(bp.BppsaError):
        bp.distil(big, big[..., :300].contiguous(), torch.zeros((1, 1, 300), dtype=torch.int32, device="cuda"))
