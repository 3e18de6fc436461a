"""The optimiser's binding: how long what a step reads and writes is kept."""
import pytest


class _Held:
    def __init__(self):
        self.recorded = []

    def record_stream(self, stream):
        self.recorded.append(stream)

    def data_ptr(self):
        return 1


class _Stream:
    def __init__(self, number):
        import torch
        self.cuda_stream, self.device = number, torch.device("cuda:0")


def test_a_step_on_another_stream_keeps_all_that_it_uses(monkeypatch):
    import torch
    from paper_1907_10134_amd import optim
    own, other, third = _Stream(7), _Stream(9), _Stream(11)
    now = [own]
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: now[-1])
    monkeypatch.setattr(optim, "_stream", lambda stream=None: (stream or now[-1]).cuda_stream)
    monkeypatch.setattr(optim, "_check", lambda *a: None)
    monkeypatch.setattr(optim._lib, "bppsa_adamw_step", lambda *a: 0)
    opt = object.__new__(optim.AdamW)
    opt.params, opt.grads, opt.copies, opt.state = [_Held(), _Held()], [_Held(), _Held()], [_Held(), _Held()], {"m": [_Held()], "v": [_Held()]}
    opt._tensors, opt._pieces, opt._n_pieces, opt._grad_type, opt._device, opt._streams, opt._readers = _Held(), _Held(), 1, 0, 0, {7}, {7}
    opt.state_bits, opt.t, opt.lr, opt.beta1, opt.beta2, opt.eps = 32, 0, 1e-3, 0.9, 0.999, 1e-8
    held = [opt._tensors, opt._pieces, *opt.params, *opt.grads, *opt.copies, *opt.state["m"], *opt.state["v"]]
    opt.step()
    assert all(x.recorded == [] for x in held)
    now.append(other)
    opt.step()
    opt.step()
    now.pop()
    assert all(x.recorded == [other] for x in held)
    opt.step(stream=third)
    opt.copies = None
    opt.step(stream=third)
    opt.step()
    assert all(x.recorded == [other, third] for x in held) and opt.t == 6


@pytest.mark.gpu
@pytest.mark.parametrize("bits", (32, 8))
def test_the_moments_of_a_dropped_optimiser_are_not_given_out_again(bits):
    """The optimiser goes before its step on the other stream has run, which reads its lists and writes its moments."""
    import torch
    import paper_1907_10134_amd as bp
    made = lambda: [torch.linspace(-1, 1, 40000, device="cuda"), torch.linspace(1, 2, 40000, device="cuda")]
    (p, g), (q, h) = made(), made()
    bp.AdamW([q], [h], state_bits=bits).step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    opt = bp.AdamW([p], [g], state_bits=bits)
    mine = [opt._tensors, opt._pieces] + [x[0] for x in opt.state.values()]
    places, sizes = {x.data_ptr() for x in mine}, [x.numel() * x.element_size() for x in mine]
    with torch.cuda.stream(side):
        busy = torch.zeros(1 << 28, device="cuda")
        for _ in range(20):
            busy += 1.0                        # some milliseconds in front of the step
    opt.step(stream=side)
    del opt, mine
    new = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(4)]      # not written: nothing may depend on it
    taken = places & {x.data_ptr() for x in new}
    side.synchronize()
    assert not taken and torch.equal(p, q)


@pytest.mark.gpu
def test_gradients_of_other_tensors_are_kept_too():
    import torch
    import paper_1907_10134_amd as bp
    p, side = torch.ones(300, device="cuda"), torch.cuda.Stream()
    opt = bp.AdamW([p], [torch.ones(300, device="cuda")])
    side.wait_stream(torch.cuda.current_stream())
    opt.step(stream=side)
    assert len(opt._streams) == len(opt._readers) == 2
    opt.read_gradients([torch.ones(300, device="cuda")])
    assert len(opt._streams) == 2 and len(opt._readers) == 1
    side.wait_stream(torch.cuda.current_stream())
    opt.step(stream=side)
    side.synchronize()
    assert len(opt._streams) == len(opt._readers) == 2 and bool((p < 1).all())
