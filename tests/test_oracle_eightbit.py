"""The oracle of the 8-bit operators against its definitions: e4m3 against the type's own table, scales by search, the norm's backward pass
against differences.  CPU only."""

import numpy as np
import pytest
import torch

from oracle import eightbit as o8


def all_e4m3():
    """The 253 finite values by the layout of the type: sign, 4 bits of exponent, 3 of fraction."""
    out = []
    for s in (1.0, -1.0):
        for e in range(16):
            for f in range(8):
                if e == 15 and f == 7:
                    continue
                out.append(s * (f * 2.0 ** -9 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7)))
    return np.array(out)


def test_e4m3_values_stay_and_their_bytes_are_the_types():
    v = all_e4m3()
    assert np.array_equal(o8.to_e4m3(v), v)
    by = o8.bits_of(v)
    back = torch.from_numpy(by).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(back.astype(np.float64), v)


def test_e4m3_rounds_to_the_nearest_and_ties_to_even():
    v = np.unique(all_e4m3())
    g = np.random.default_rng(1)
    x = np.concatenate([g.uniform(-448, 448, 4000), g.normal(0, 0.01, 4000), (v[1:] + v[:-1]) / 2])
    q = o8.to_e4m3(x)
    near = np.min(np.abs(x[:, None] - v[None]), axis=1)
    assert np.array_equal(np.abs(q - x), near)
    ties = (v[1:] + v[:-1]) / 2
    assert np.all(o8.bits_of(o8.to_e4m3(ties)) % 2 == 0)
    assert np.array_equal(torch.from_numpy(x).float().to(torch.float8_e4m3fn).float().numpy(), o8.to_e4m3(x.astype(np.float32).astype(np.float64)))


@pytest.mark.parametrize("block", [1, 128])
def test_scales_are_the_least_that_fit(block):
    g = np.random.default_rng(2)
    x = g.normal(0, 1, (130, 300)) * 10.0 ** g.integers(-30, 30, (130, 1))
    x[3] = 0
    x[4, :] = 448.0
    x[5, :] = np.nextafter(448.0, 449)
    x[6, :] = 1e-45
    e = o8.exponents(x, block)
    for i in range(e.shape[0]):
        for j in range(e.shape[1]):
            big = np.abs(x[i * block:(i + 1) * block, j * 128:(j + 1) * 128]).max()
            assert big <= 448 * 2.0 ** e[i, j] and (e[i, j] == -127 or big > 448 * 2.0 ** (e[i, j] - 1))
    q, e = o8.quantize(x, block)
    step = np.maximum(np.abs(x), 2.0 ** (o8.spread(e, block, x.shape) - 6.0)) / 8
    assert np.all(np.abs(o8.dequantize(q, e, block) - x) <= step / 2)


def test_norm_backward_against_differences():
    g = np.random.default_rng(3)
    h, gamma, dy = g.normal(0, 2, (3, 7)), g.normal(1, 0.2, 7), g.normal(0, 1, (3, 7))
    dx, dgamma = o8.rmsnorm_backward(dy, h, gamma, 1e-3)
    loss = lambda h, gamma: np.sum(dy * o8.rmsnorm(h, gamma, 1e-3)[0])  # noqa: E731
    d = 1e-6
    for i in range(3):
        for j in range(7):
            p, m = h.copy(), h.copy()
            p[i, j] += d
            m[i, j] -= d
            assert abs((loss(p, gamma) - loss(m, gamma)) / (2 * d) - dx[i, j]) < 1e-8
    for j in range(7):
        p, m = gamma.copy(), gamma.copy()
        p[j] += d
        m[j] -= d
        assert abs((loss(h, p) - loss(h, m)) / (2 * d) - dgamma[j]) < 1e-8
    assert np.array_equal(o8.rmsnorm_backward(dy, h, gamma, 1e-3, dh=h)[0], dx + h)


def test_product_and_clip_by_hand():
    a, b = np.array([[1.0, 2.0]]), np.array([[3.0, -1.0], [-4.0, 0.5]])
    assert np.array_equal(o8.product(a, b, bias=[0.5, 0.0], relu=True), [[1.5, 0.0]])
    norm, (x, y) = o8.clip([np.array([3.0]), np.array([[4.0]])], 2.5)
    assert norm == 5.0 and abs(x[0] - 1.5) < 1e-6 and abs(y[0, 0] - 2.0) < 1e-6
    assert o8.clip([np.array([3.0])], 4.0)[1][0][0] == 3.0
