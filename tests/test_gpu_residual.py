"""The residual segment in 8 bits: its gradients beside the oracle's operators put together in the same way, and training through a frozen right
partition."""

import numpy as np
import pytest
import torch

from oracle import eightbit as o8
from paper_2403_11204_amd import api, datagen, pipeline
from paper_2403_11204_amd.residual import ResidualSegment

pytestmark = pytest.mark.gpu
DEV = "cuda"


def bf16(x):
    return torch.from_numpy(np.asarray(x, dtype=np.float64)).to(torch.bfloat16).double().numpy()


def eight(x, block):
    """What x stands for once it is in 8 bits."""
    return o8.dequantize(*o8.quantize(x, block), block)


def reference(seg, X, d):
    """(output, gradients of X and of the parameters) in float64, rounded where the segment stores a value."""
    f64 = lambda t: t.detach().double().cpu().numpy()  # noqa: E731
    h, f, kept = f64(X), None, []
    for b in seg.blocks:
        h = h if f is None else bf16(h + f)
        y, n = o8.rmsnorm(h, f64(b.gamma), seg.eps)
        w1, w2 = eight(f64(b.w1), 128), eight(f64(b.w2), 128)
        z = bf16(o8.product(eight(y, 1), w1, f64(b.b1), relu=True))
        f = bf16(o8.product(eight(z, 1), w2, f64(b.b2)))
        kept.append((h, y, z, w1, w2))
    out = bf16(h + f)
    d, grads = f64(d), []
    for b, (h, y, z, w1, w2) in zip(reversed(seg.blocks), reversed(kept)):
        da = bf16(eight(d, 1) @ w2)
        dw2 = eight(d.T, 1) @ eight(z.T, 1).T
        dz = np.where(z > 0, da, 0.0)
        dy = bf16(eight(dz, 1) @ w1)
        dw1 = eight(dz.T, 1) @ eight(bf16(y).T, 1).T
        db2, db1 = d.sum(0), dz.sum(0)
        d, dgamma = o8.rmsnorm_backward(dy, h, f64(b.gamma), seg.eps, dh=d)
        d = bf16(d)
        grads = [dgamma, dw1, db1, dw2, db2] + grads
    return out, [d] + grads


@pytest.mark.parametrize("rows,width,hidden,blocks", [(1, 64, 130, 1), (70, 200, 300, 2), (300, 512, 1024, 2)])
def test_gradients(rows, width, hidden, blocks):
    g = torch.Generator().manual_seed(rows)
    seg = ResidualSegment(width, hidden, blocks, seed=3)
    X, d = (torch.randn(rows, width, generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    out, grads = reference(seg, X, d)
    # Both sides round at the same places; where their float32 and float64 values lie on two sides of a tie they differ by a unit there, 2^-8 of a
    # bf16 value.  Were every one of the 4 values stored on the longest path of a block off by that, all one way, the two blocks' 8 would come to 2^-5.
    assert np.linalg.norm(seg.forward(X).double().cpu().numpy() - out) <= 2.0 ** -5 * np.linalg.norm(out)
    dx, got = seg.backward(X, d)
    for a, b in zip([dx] + got, grads):
        a = a.double().cpu().numpy()
        assert a.shape == b.shape and np.linalg.norm(a - b) <= 2.0 ** -5 * np.linalg.norm(b), (b.shape, np.linalg.norm(a - b) / np.linalg.norm(b))


def test_the_gradient_points_where_the_unrounded_network_does():
    """Beside differentiation of the network without any rounding: a value in 8 bits is off by 2.6 % in the mean square, so directions are near."""
    seg = ResidualSegment(128, 256, 2, seed=4)
    g = torch.Generator().manual_seed(1)
    X, d = (torch.randn(200, 128, generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    x = X.double().cpu().requires_grad_()
    params = [p.data.double().cpu().requires_grad_() for p in seg.parameters]
    h = x
    for i in range(2):
        gamma, w1, b1, w2, b2 = params[5 * i:5 * i + 5]
        n = h / torch.sqrt((h * h).mean(1, keepdim=True) + seg.eps) * gamma
        h = h + torch.relu(n @ w1.t() + b1) @ w2.t() + b2
    h.backward(d.double().cpu())
    dx, got = seg.backward(X, d)
    for a, b in zip([dx] + got, [x.grad] + [p.grad for p in params]):
        assert float(torch.nn.functional.cosine_similarity(a.double().cpu().flatten(), b.flatten(), dim=0)) > 0.9


def test_training_through_a_frozen_partition():
    n, width, classes = 512, 256, 10
    X, y = datagen.blob_images(n, classes, 16, seed=2)
    X = torch.from_numpy(X).to(DEV).to(torch.bfloat16)
    y = torch.from_numpy(y).to(DEV)
    assert X.shape[1] == width
    left = ResidualSegment(width, 384, 2, lr=0.05, momentum=0.9, max_norm=1.0)
    right = api.Segment([width, 64, classes], api.RELU_HIDDEN_IDENTITY_LAST, api.SOFTMAX_XENT, max_batch=128, dtype=api.BF16, input_grad=True)
    right.init(5)
    before = [p.data.clone() for p in left.parameters]
    frozen = right.get_params(0)[0].clone()
    losses = pipeline.recovery_epochs(left, right, X, y, epochs=6, batch=128)
    assert losses[-1] < 0.6 * losses[0], losses
    assert all(not torch.equal(p.data, q) for p, q in zip(left.parameters, before)) and torch.equal(right.get_params(0)[0], frozen)
    assert pipeline.accuracy([left, right], X, y, batch=100) > 0.5
    # not finite: nothing changes
    before = [p.data.clone() for p in left.parameters]
    bad = torch.zeros(8, width, dtype=torch.bfloat16, device=DEV)
    bad[3, 4] = float("inf")
    left.step_external(X[:8], bad)
    assert not np.isfinite(float(left.gradient_norm)) and all(torch.equal(p.data, q) for p, q in zip(left.parameters, before))
