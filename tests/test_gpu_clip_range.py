"""Clipping where the factor, or the norm, leaves float32's range.  Tolerances as for clipping elsewhere: 3 u of a value with u = 2^-24, 2^-149 where it
leaves float32's range, 2^-8 for rounding to bf16."""

import numpy as np
import pytest
import torch

from oracle import eightbit as o8
from paper_2403_11204_amd import api

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("values,max_norm", [([1e38, -3e37, 1e30], 1e-20), ([1e30, 5e29, -1e22], 1e-12), ([3e37, -1e37], 1e-9), ([1e20, 1e3], 1e-25), ([3.0, 4.0], 1e-38), ([1e38], 1e-44)])
def test_a_factor_below_the_range_of_float32(values, max_norm, dtype):
    """The values themselves are in its range."""
    max_norm = float(np.float32(max_norm))
    t = torch.tensor(values).to(dtype).to(DEV)
    norm, (ref,) = o8.clip([f64(t)], max_norm)
    out = [torch.empty_like(t)]
    assert abs(float(api.clip_gradients([t], max_norm, out=out)) - norm) <= 2 * U * norm
    assert np.all(np.abs(f64(out[0]) - ref) <= (3 * U + (2.0 ** -8 if dtype is torch.bfloat16 else 0)) * np.abs(ref) + 2.0 ** (-149 if dtype is torch.float32 else -133)), (f64(out[0]), ref)
    api.clip_gradients([t], max_norm)
    assert torch.equal(t, out[0])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_norm_that_float32_does_not_hold_leaves_the_values(dtype):
    """What the caller is given is infinite: that the step is to be skipped, and that nothing has been scaled."""
    t = [torch.tensor([3e38, -3e38, 5.0]).to(dtype).to(DEV), torch.arange(7.0).to(dtype).to(DEV)]
    before, out = [x.clone() for x in t], [torch.empty_like(x) for x in t]
    assert float(api.gradient_norm(t)) == float("inf") == float(api.clip_gradients(t, 1.0, out=out))
    assert all(torch.equal(a, b) for a, b in zip(out, before))
    assert float(api.clip_gradients(t, 1.0)) == float("inf") and all(torch.equal(a, b) for a, b in zip(t, before))
    # the largest norm that it holds
    big = torch.tensor([3.4e38], device=DEV)
    norm = float(api.clip_gradients([big], 2.0))
    assert np.isfinite(norm) and abs(float(big) - 2.0) <= 4 * U * 2.0
