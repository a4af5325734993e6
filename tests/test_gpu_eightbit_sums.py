"""How exactly products of 8-bit matrices are added, in both forms.

With p the products of one output, G the groups of 8 consecutive k and u = 2^-24:
  float32 sums   (float32 outputs, bf16 outputs that ask for them, few rows) exact products, added in float32 in any order: (K + 2) u sum|p|
  the scaled matrix instruction (bf16 outputs of many rows)  in each group the products are cut off at a multiple of 2^-13 2^(the sum of the largest one's
                 exponents), which is 2^-13 of the largest product at most: the largest itself loses nothing (its factors have 4 bits each), the other seven less than that each.  The
                 groups' sums are added with 24 bits and cut off, not rounded: one unit, 2 u, each time.  7 2^-13 sum over G of max|p| + (K + 2) 2 u sum|p|
and 2^-8 of the result for rounding it to bf16.
"""

import numpy as np
import pytest
import torch

from paper_2403_11204_amd import api

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24


def eight(x, block=1):
    """A matrix of e4m3 values as an 8-bit one, scales 1."""
    m = api.empty_quantized(*x.shape, block)
    full = m.q.view(torch.uint8).as_strided((x.shape[0], m.q.stride(0)), (m.q.stride(0), 1))
    full.zero_()
    m.q.copy_(x.to(torch.float8_e4m3fn))
    m.scales.view(torch.uint8).fill_(127)
    return m


def e4m3(x):
    return x.clamp(-448, 448).to(torch.float8_e4m3fn).float()


def cancelling(m, n, k, seed):
    """e4m3 matrices spread over many powers of two whose products cancel: the second half of the contraction takes back the first but for one small value."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    half = k // 2

    def spread(rows):
        return e4m3(torch.randn(rows, half, device=DEV, generator=g) * torch.exp(1.5 * torch.randn(rows, half, device=DEV, generator=g)))

    a, b = spread(m), spread(n)
    small = e4m3(0.01 * torch.randn(m, 2 * half, device=DEV, generator=g))
    a = torch.cat([a, -a], 1)
    a = torch.where(torch.rand(a.shape, device=DEV, generator=g) < 0.02, small, a)
    return a, torch.cat([b, b], 1)


def sizes(a, b):
    """(the products' sums, of their magnitudes, of the largest of each 8) in float64."""
    p64, s64 = a.double() @ b.double().t().contiguous(), a.abs().double() @ b.abs().double().t().contiguous()
    most = torch.zeros_like(p64)
    for k in range(0, a.shape[1], 8):
        most += (a[:, None, k:k + 8] * b[None, :, k:k + 8]).abs().amax(2).double()
    return p64, s64, most


# tiles in one group, two and four of wavefronts, split, and the 256x256 kernel
@pytest.mark.parametrize("m,n,k", [(40, 48, 128), (64, 80, 16), (100, 130, 384), (65, 65, 3000), (600, 500, 256), (64, 64, 16384), (3000, 3104, 128)])
def test_sums_whose_terms_cancel(m, n, k):
    a, b = cancelling(m, n, k, m + k)
    p64, s64, most = sizes(a, b)
    x, y = eight(a), eight(b)
    tight = (k + 2) * U * s64
    assert bool(((api.product(x, y, dtype=api.F32).double() - p64).abs() <= tight).all())
    assert bool(((api.product(x, y, float32_sums=True).double() - p64).abs() <= tight + 2.0 ** -8 * (p64.abs() + tight)).all())
    loose = 7 * 2.0 ** -13 * most + (k + 2) * 2 * U * s64
    assert bool(((api.product(x, y).double() - p64).abs() <= loose + 2.0 ** -8 * (p64.abs() + loose)).all())


@pytest.mark.parametrize("m", [1, 3, 20, 32, 40, 300])
def test_what_a_product_of_eight_neighbours_may_lose(m):
    """65536 - 65536 + 7: float32 sums keep the 7 wherever it stands; the scaled instruction does where it is not one of the eight beside a large one."""
    a, b = torch.zeros(m, 256, device=DEV), torch.zeros(70, 256, device=DEV)
    a[:, 0], a[:, 100], a[:, 5], b[:, 0], b[:, 100], b[:, 5] = 256, -256, 7, 256, 256, 1
    out = torch.empty(m, 70, dtype=torch.bfloat16, device=DEV)
    assert bool((api.product(eight(a), eight(b), float32_sums=True) == 7).all())
    assert bool((api.product(eight(a), eight(b), out=out, float32_sums=True) == 7).all()) and bool((out == 7).all())
    assert bool((api.product(eight(a), eight(b), dtype=api.F32) == 7).all())
    a[:, 5], a[:, 50], b[:, 5], b[:, 50] = 0, 512 * 0.5, 0, 1
    assert bool((api.product(eight(a), eight(b)) == 256).all())


@pytest.mark.parametrize("n,k", [(130, 784), (512, 4100)])
def test_a_row_alone_and_in_a_batch_with_float32_sums(n, k):
    g = torch.Generator(device=DEV)
    g.manual_seed(n)
    x, w = torch.randn(300, k, device=DEV, generator=g), torch.randn(n, k, device=DEV, generator=g)
    x8, w8 = api.quantize(x).rows, api.quantize(w, block=128).rows
    whole = api.product(x8, w8, float32_sums=True).double()
    s = x8.scales.float().repeat_interleave(128, 1)[:, :k]
    t = w8.scales.float().repeat_interleave(128, 0)[:n].repeat_interleave(128, 1)[:, :k]
    size = (x8.q.float() * s).abs().double() @ (w8.q.float() * t).abs().double().t().contiguous()
    for r in (0, 7, 299):
        one = api.product(api.Quantized(x8.q[r:r + 1], x8.scales[r:r + 1], 1), w8).double()
        assert bool(((one - whole[r:r + 1]).abs() <= 2 * (k + 2) * U * size[r:r + 1] + 2.0 ** -7 * one.abs()).all())


def test_float32_sums_of_large_products_are_the_float32_outputs_rounded():
    """The 256x256 kernel, whole and ragged, dense and into a wider matrix: the same sums, rounded once."""
    for m, n, k in ((4096, 4096, 400), (4000, 4100, 300)):
        g = torch.Generator(device=DEV)
        g.manual_seed(k)
        x = api.quantize(torch.randn(m, k, device=DEV, generator=g)).rows
        y = api.quantize(torch.randn(n, k, device=DEV, generator=g), block=128).rows
        ref = api.product(x, y, dtype=api.F32).to(torch.bfloat16)
        assert torch.equal(api.product(x, y, float32_sums=True), ref)
        room = torch.full((m, n + 3), 7.0, dtype=torch.bfloat16, device=DEV)
        api.product(x, y, out=room[:, 1:n + 1], float32_sums=True)
        assert torch.equal(room[:, 1:n + 1], ref) and bool((room[:, 0] == 7).all()) and bool((room[:, n + 1:] == 7).all())
