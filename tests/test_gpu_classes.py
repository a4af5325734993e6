"""The operators of a last layer over many classes put together: trained, distilled from a teacher served in integers, as a frozen right partition, joined."""

import os
import re

import numpy as np
import pytest
import torch

from oracle import class_loss, integers
from paper_2403_11204_amd import api, pipeline
from paper_2403_11204_amd.classes import ClassLayer
from paper_2403_11204_amd.residual import ResidualSegment

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _np(t):
    return t.detach().cpu().double().numpy()


def _off(got, want, tol):
    assert (np.abs(_np(got) - want) <= tol).all(), float((np.abs(_np(got) - want) - tol).max())


def _rows(seed, n, width):
    return torch.randn(n, width, generator=torch.Generator().manual_seed(seed)).bfloat16().cuda()


def test_step_is_sgd_with_the_gradients():
    layer = ClassLayer(64, 300, lr=0.5, momentum=0.9, seed=1)
    x = _rows(1, 90, 64)
    y = torch.randint(-1, 300, (90,), dtype=torch.int32, generator=torch.Generator().manual_seed(2)).cuda()
    w, b, vw, vb = _np(layer.w), _np(layer.b), 0.0, 0.0
    for _ in range(2):
        o = class_loss.loss(_np(x), _np(layer.w16), y.cpu().numpy()[:, None], bias=_np(layer.b))
        loss = layer.step(x, y)
        vw, vb = 0.9 * vw + o["dw"], 0.9 * vb + o["dbias"]
        w, b = w - 0.5 * vw, b - 0.5 * vb
        # logits below 8 off by 6 sqrt(64) 2^-24 8, so P by 2^-13 of it, rounded to bf16: 2^-8 of each of 90 terms; two steps add up, 0.9 of the first one's once more
        size = np.abs(o["dz"]).T @ np.abs(_np(x))
        assert abs(float(loss) - o["loss"]) < 1e-4
        _off(layer.w, w, 0.5 * 3 * 1.05 * 2.0 ** -8 * size + 1e-6)
        _off(layer.b, b, 0.5 * 3 * 2.0 ** -12 * np.abs(o["dz"]).sum(0) + 1e-6)
        assert torch.equal(layer.w16, layer.w.data.bfloat16())
        w, b = _np(layer.w), _np(layer.b)          # (the next step starts from what is there)


def test_teacher_in_integers_distilled():
    """A teacher's logits computed in integers, its best classes, a student's step against them: all calls in a row, then the same replayed from a graph."""
    teacher, student = ClassLayer(64, 500, seed=3), ClassLayer(64, 500, lr=0.1, momentum=0.0, seed=4)
    x = _rows(5, 70, 64)
    z = teacher.forward(x)
    q, s = integers.quantize(_np(x))
    wq, ws = integers.quantize(_np(teacher.w))
    want = integers.product(q, s, wq, ws, _np(teacher.b))
    _off(z, want, 1.01 * 2.0 ** -8 * np.abs(want) + 2.0 ** -21 * np.abs(want).max())
    top, ids = z.topk(8, 1)
    o = class_loss.loss(_np(x), _np(student.w16), ids.cpu().numpy(), _np(top), _np(student.b), 2.0)
    w = _np(student.w)
    loss = student.distil(x, top, ids, temperature=2.0)
    assert abs(float(loss) - o["loss"]) < 1e-4
    _off(student.w, w - 0.1 * o["dw"], 0.1 * 1.05 * 2.0 ** -8 * (np.abs(o["dz"]).T @ np.abs(_np(x))) + 1e-6)

    w8 = api.quantize_integers(teacher.w.data)

    def run():
        z = api.product_integers(api.quantize_integers(x), w8, bias=teacher.b.data)
        top, ids = z.topk(8, 1)
        r = api.linear_distillation(x, student.w16, top, ids, bias=student.b.data, temperature=2.0)
        c = api.linear_cross_entropy(x, student.w16, ids[:, 0].contiguous(), bias=student.b.data)
        return list(r) + list(c)

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = run()
    for seed in range(3):
        x.copy_(_rows(10 + seed, 70, 64))
        graph.replay()
        eager = run()
        torch.cuda.synchronize()
        for u, v in zip(captured, eager):
            assert torch.equal(u, v)


def test_gradients_clipped_together():
    layer = ClassLayer(48, 200, seed=6)
    r = api.linear_cross_entropy(_rows(7, 33, 48), layer.w16, torch.arange(33, device=DEV), bias=layer.b.data, dtype=api.F32)
    grads = [r.dw, r.dbias]
    want = torch.sqrt(sum((g.double() ** 2).sum() for g in grads))
    norm = api.clip_gradients(grads, 0.5 * float(want))
    assert abs(float(norm) - float(want)) <= 2.0 ** -22 * float(want)
    assert abs(float(api.gradient_norm(grads)) - 0.5 * float(want)) <= 2.0 ** -20 * float(want)


def test_right_partition():
    """Frozen behind a residual left partition, joined with it, trained on its stored response."""
    left, right = ResidualSegment(128, 160, 1, seed=8), ClassLayer(128, 700, seed=9)
    X = _rows(11, 150, 128)
    y = torch.randint(0, 700, (150,), dtype=torch.int32, generator=torch.Generator().manual_seed(12)).cuda()
    resp = left.forward(X)
    dx, loss = right.input_grad(resp, y)
    o = class_loss.loss(_np(resp), _np(right.w16), y.cpu().numpy()[:, None], bias=_np(right.b))
    assert abs(float(loss) - o["loss"]) < 1e-4
    _off(dx, o["dx"], 1.05 * 2.0 ** -8 * (np.abs(o["dz"]) @ np.abs(_np(right.w16))) + 1.01 * 2.0 ** -8 * np.abs(o["dx"]) + 1e-8)
    before = right.w.data.clone()
    losses = pipeline.recovery_epochs(left, right, X, y, epochs=2, batch=64)
    assert len(losses) == 2 and all(np.isfinite(losses)) and torch.equal(before, right.w.data)
    stored = pipeline.store_response(left, X, batch=64)
    losses = pipeline.train_epochs(right, stored, y, epochs=2, batch=64)
    assert len(losses) == 2 and all(np.isfinite(losses)) and not torch.equal(before, right.w.data)
    z = pipeline.joined_forward([left, right], X, batch=64)
    assert torch.equal(z, torch.cat([right.forward(left.forward(X[a:a + 64])) for a in range(0, 150, 64)]))
    hits = pipeline.accuracy([left, right], X, y, batch=64)
    assert hits == (_np(z).argmax(1) == y.cpu().numpy()).mean()                    # (numpy's is the first among equals)


def test_the_readmes_example():
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")).read()
    block = re.search(r"\n\n((?:    .*\n)*    r = api\.linear_cross_entropy(?:.*\n)(?:    .*\n)*)", text).group(1)
    x, V, b = _rows(21, 70, 200), _rows(22, 500, 200) / 16, _rows(23, 1, 500)[0].float()
    y = torch.randint(-40, 500, (70,), dtype=torch.int32, generator=torch.Generator().manual_seed(24)).cuda()
    teacher = _rows(25, 70, 500)
    have = {"api": api, "x": x, "V": V, "b": b, "y": y, "teacher_logits": teacher}
    exec(re.sub(r"^    ", "", block, flags=re.M), have)
    top, ids = teacher.topk(32, 1)
    o = class_loss.loss(_np(x), _np(V), y.cpu().numpy()[:, None], bias=_np(b))
    od = class_loss.loss(_np(x), _np(V), ids.cpu().numpy(), _np(top), _np(b), 2.0)
    # logits below 16: 200 additions' 2^-24 of it come to 2e-4 at the most, of random sign to 1.4e-5; twice that, 4 times with the temperature squared
    assert abs(float(have["r"].loss) - o["loss"]) < 1e-4 and abs(float(have["d"].loss) - od["loss"]) < 1e-4
    _off(have["r"].dx, o["dx"], 1.05 * 2.0 ** -8 * (np.abs(o["dz"]) @ np.abs(_np(V))) + 1.01 * 2.0 ** -8 * np.abs(o["dx"]) + 1e-8)
    # an integer is half a scale off
    X, W = _np(x), _np(V)
    sx, sw = np.abs(X).max(1)[:, None] / 127, np.abs(W).max(1)[:, None] / 127
    tol = (sx / 2 * np.abs(W).sum(1) + np.abs(X).sum(1)[:, None] * sw.T / 2 + 200 * sx * sw.T / 4) * (1 + 2.0 ** -20)
    z = X @ W.T + _np(b)
    _off(have["z"], z, tol * (1 + 2.0 ** -8) + 1.01 * 2.0 ** -8 * np.abs(z))
