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

    def quantize_integers(self, x):
        self.quantized.append(x)
        s = x.float().abs().amax(1) / 127
        return api.Integers((x.float() / s[:, None]).round().to(torch.int8), s)

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
