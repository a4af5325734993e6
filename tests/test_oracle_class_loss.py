"""The oracle of the losses over a linear layer's classes against differences and closed forms.  CPU only."""

import numpy as np
import pytest

from oracle import class_loss


def _case(seed, rows=4, classes=7, dim=5, k=3):
    g = np.random.default_rng(seed)
    x, w, b = g.normal(size=(rows, dim)), g.normal(size=(classes, dim)), g.normal(size=classes)
    ids = np.stack([g.permutation(classes)[:k] for _ in range(rows)])
    top = g.normal(size=(rows, k)) * 2
    return x, w, b, ids, top


@pytest.mark.parametrize("teacher,temperature", [(False, 1.0), (True, 1.0), (True, 3.0)])
def test_gradients_are_the_differences(teacher, temperature):
    x, w, b, ids, top = _case(3)
    ids[1] = -1                              # a row that does not count
    if teacher:
        ids[2, 1] = ids[2, 0]                # a class twice
        top[3, 0] = -np.inf
    args = dict(classes=ids if teacher else ids[:, :1], top=top if teacher else None, temperature=temperature, scale=1.5)
    r = class_loss.loss(x, w, bias=b, **args)
    h = 1e-5
    for name, a in (("dx", x), ("dw", w), ("dbias", b)):
        for at in np.ndindex(a.shape):
            keep = a[at]
            a[at] = keep + h
            up = class_loss.loss(x, w, bias=b, **args)["loss"]
            a[at] = keep - h
            down = class_loss.loss(x, w, bias=b, **args)["loss"]
            a[at] = keep
            # central differences: h^2 / 6 of the third derivative (some 10 here) and 2^-52 of the loss over h
            assert abs(1.5 * (up - down) / (2 * h) - r[name][at]) < 1e-8, (name, at)


def test_closed_forms():
    x, w = np.zeros((2, 3)), np.zeros((4, 3))
    r = class_loss.loss(x, w, np.array([[1], [9]]))
    assert r["loss"] == pytest.approx(np.log(4)) and list(r["counts"]) == [True, False]
    assert np.allclose(r["dz"], [[0.25, -0.75, 0.25, 0.25], [0, 0, 0, 0]])
    # a teacher equal to the student over all classes: no divergence, no gradient
    x, w, b, _, _ = _case(5)
    ids = np.tile(np.arange(7), (4, 1))
    r = class_loss.loss(x, w, ids, top=x @ w.T + b, bias=b, temperature=2.0)
    assert abs(r["loss"]) < 1e-14 and np.abs(r["dz"]).max() < 1e-15
