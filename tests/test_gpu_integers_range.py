"""Products of integers whose scales are far from 1: what leaves float32's range is the result, never a step on the way.

The sum goes to float32 (2^-24 of it), times a scale (2^-24; below 2^-126 exact, since it is an integer), times the other and plus the bias (2^-24 of the product and of the result,
below 2^-126 half of 2^-149)."""

import numpy as np
import pytest
import torch

from paper_2403_11204_amd import api

pytestmark = pytest.mark.gpu

# few rows, tiles (one part and parts joined), 256x256 tiles whole and ragged
SHAPES = [(2, 100, 300), (40, 600, 64), (64, 64, 16384), (300, 500, 1000), (3000, 3000, 304), (3000, 3001, 300)]
EXTREMES = torch.tensor([2.4e30, 2.6e36, 1e-38, 1e-42, 1.4e-45, 1.0, 0.0, 3.3e-10, 1e25])


def _matrix(seed, rows, k, scales):
    g = torch.Generator().manual_seed(seed)
    m = api.quantize_integers(torch.zeros(rows, k, device="cuda"))
    m.q.copy_(torch.randint(-128, 128, (rows, k), generator=g, dtype=torch.int8))
    m.scales.copy_(scales)
    return m


def _check(got, a, b, bias, half):
    sums = a.q.double() @ b.q.double().t()
    prod = sums * a.scales.double()[:, None] * b.scales.double()
    want = prod + bias.double()
    most = float(torch.finfo(torch.float32).max)
    inside = want.abs() < most * (1 - 2.0 ** -8)
    off = (got.double() - want).abs() - (3.01 * 2.0 ** -24 * prod.abs() + 2.0 ** -24 * want.abs() + half * want.abs() + 2.0 ** -149 + (2.0 ** -133 if half else 0))
    assert (off[inside] <= 0).all(), float(off[inside].max())
    beyond = want.abs() > most * (1 + 2.0 ** -8)
    assert (got[beyond].double() == torch.sign(want[beyond]) * float("inf")).all()
    assert not got.isnan().any()


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_scales_far_from_one(m, n, k, dtype):
    i, j = torch.arange(m) % len(EXTREMES), torch.arange(n) % len(EXTREMES)
    a, b = _matrix(1, m, k, EXTREMES[i]), _matrix(2, n, k, EXTREMES[j])
    bias = torch.randn(n, generator=torch.Generator().manual_seed(3)).cuda()
    bias[::2] = 0
    half, dt = (0.0, api.F32) if dtype == "fp32" else (1.01 * 2.0 ** -8, api.BF16)
    _check(api.product_integers(a, b, bias=bias, dtype=dt), a, b, bias, half)
    _check(api.product_integers(a, b, dtype=dt), a, b, torch.zeros_like(bias), half)


def test_a_layer_of_large_rows():
    """Rows near 1e33 and weights near 1e-10, as they come from quantising: every result is a number."""
    g = torch.Generator().manual_seed(5)
    x, w = (torch.rand(40, 16384, generator=g) + 0.5).cuda() * 1e33, (torch.rand(70, 16384, generator=g) + 0.5).cuda() * 1e-10
    a, b = api.quantize_integers(x), api.quantize_integers(w)
    _check(api.product_integers(a, b, dtype=api.F32), a, b, torch.zeros(70, device="cuda"), 0.0)
    assert np.isfinite(api.product_integers(a, b, dtype=api.F32).cpu().numpy()).all()
