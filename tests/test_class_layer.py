"""What ClassLayer keeps and when it writes it: on the CPU against a stand-in for the library's calls, on the device on several streams."""

import types

import pytest
import torch

from paper_2403_11204_amd import api, classes


class Calls:
    """Stands in for api: plain torch, and a list of what was quantised."""

    BF16, F32 = api.BF16, api.F32

    def __init__(self):
        self.quantized = []

    def quantize_integers(self, x, out=None):
        self.quantized.append(x)
        s = x.float().abs().amax(1) / 127
        r = api.Integers((x.float() / s[:, None]).round().to(torch.int8), s)
        if out is not None:
            out.q.copy_(r.q), out.scales.copy_(r.scales)
        return out or r

    def product_integers(self, a, b, bias=None, out=None):
        return (a.q.float() * a.scales[:, None]) @ (b.q.float() * b.scales[:, None]).t() + bias


@pytest.fixture
def calls(monkeypatch):
    c = Calls()
    monkeypatch.setattr(classes, "api", c)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: types.SimpleNamespace(synchronize=lambda: None))
    return c


def test_forward_writes_nothing_that_is_kept(calls):
    """The weights' integers are there before the first forward, which quantises its rows and nothing else."""
    layer = classes.ClassLayer(8, 20, device="cpu")
    assert len(calls.quantized) == 1 and calls.quantized[0].data_ptr() == layer.w.data_ptr()
    kept = {k: id(v) for k, v in vars(layer).items()}
    x = torch.randn(3, 8).bfloat16()
    for _ in range(2):
        layer.forward(x)
    assert [t is x for t in calls.quantized[1:]] == [True, True] and kept == {k: id(v) for k, v in vars(layer).items()}
    layer.w.data.mul_(2)
    layer.refresh()
    assert torch.equal(layer._w8.scales, layer.w.data.abs().amax(1) / 127)


def _places(layer):
    state = [v for p in (layer.w, layer.b) for v in layer.optimizer.state[p].values() if torch.is_tensor(v)]
    return [t.data_ptr() for t in [layer.w, layer.b, layer.w16, *layer._w8, *state]]


def test_copies_stay_where_they_are(calls):
    layer = classes.ClassLayer(8, 20, device="cpu")
    places = _places(layer)
    assert len(places) == 7                                  # momentum is there before the first step
    layer.w.grad, layer.b.grad = torch.ones_like(layer.w), torch.ones_like(layer.b)
    w = layer.w.data.clone()
    layer.optimizer.step()
    assert torch.equal(layer.w.data, w - 0.01)               # zeros times 0.9 and the gradient
    layer.refresh()
    assert places == _places(layer) and torch.equal(layer.w16, layer.w.data.bfloat16()) and torch.equal(layer._w8.scales, layer.w.data.abs().amax(1) / 127)


@pytest.mark.gpu
def test_served_on_two_streams():
    """A new layer, and one that has just been trained, on streams that have not waited for each other's first call."""
    streams = [torch.cuda.Stream() for _ in range(2)]
    g = torch.Generator().manual_seed(1)
    x = torch.randn(40, 512, generator=g).bfloat16().cuda()
    y = torch.randint(20000, (40,), generator=g).cuda()
    torch.cuda.synchronize()
    layer = classes.ClassLayer(512, 20000, lr=1.0, seed=1)

    def serve():
        got = []
        for s in streams:
            with torch.cuda.stream(s):
                got.append((layer.forward(x), layer.input_grad(x, y)[0]))
        torch.cuda.synchronize()
        want = layer.forward(x), layer.input_grad(x, y)[0]
        for both in got:
            assert all(torch.equal(u, v) for u, v in zip(both, want))
        return want

    before = serve()
    layer.step(x, y)
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    assert not torch.equal(serve()[0], before[0])


@pytest.mark.gpu
@pytest.mark.parametrize("momentum", [0.9, 0.0])
def test_captured_steps_and_forwards(momentum):
    """A training step and a forward, each in a graph of its own and the first that the layer does, replayed between eager ones: every one works on the parameters as they are then."""
    def batch(seed):
        g = torch.Generator().manual_seed(seed)
        return torch.randn(70, 96, generator=g).bfloat16().cuda(), torch.randint(-1, 600, (70,), generator=g).cuda()

    x, y = batch(1)
    captured, eager = (classes.ClassLayer(96, 600, lr=0.5, momentum=momentum, seed=2) for _ in range(2))
    api.product_integers(api.quantize_integers(x), captured._w8)          # (the library is loaded)
    api.linear_cross_entropy(x, captured.w16, y, bias=captured.b.data, dtype=api.F32)
    torch.cuda.synchronize()
    step, forward = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(forward):
        z = captured.forward(x)
    with torch.cuda.graph(step):
        loss = captured.step(x, y)
    places = _places(captured)
    for i in range(5):
        xi, yi = batch(10 + i)
        x.copy_(xi), y.copy_(yi)
        if i == 3:                                   # an eager one among them
            losses = captured.step(x, y), eager.step(x, y)
        else:
            step.replay()
            losses = loss, eager.step(x, y)
        forward.replay()
        want = eager.forward(x)
        torch.cuda.synchronize()
        assert torch.equal(*losses) and torch.equal(z, want) and torch.equal(captured.forward(x), want), i
        assert torch.equal(captured.w, eager.w) and torch.equal(captured.b, eager.b) and torch.equal(captured.w16, eager.w16), i
    assert places == _places(captured)
