"""Products of 8-bit matrices at their edges: what lies past the last column, ragged sides on every kernel."""

import pytest
import torch

from paper_2403_11204_amd import api

pytestmark = pytest.mark.gpu
DEV = "cuda"


def integers(rows, cols, block, seed, past):
    """(an 8-bit matrix of integers -4 .. 4 at scales of 1/2 .. 2 whose memory past the last column holds the byte `past`, the float64 matrix)."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    m = api.empty_quantized(rows, cols, block)
    m.q.view(torch.uint8).as_strided((rows, m.q.stride(0)), (m.q.stride(0), 1)).fill_(past)
    x = torch.randint(-4, 5, (rows, cols), device=DEV, generator=g).float()
    m.q.copy_(x.to(torch.float8_e4m3fn))
    e = torch.randint(126, 129, m.scales.shape, device=DEV, generator=g)
    m.scales.view(torch.uint8).copy_(e.to(torch.uint8))
    s = torch.exp2((e - 127).double()).repeat_interleave(block, 0)[:rows].repeat_interleave(128, 1)[:, :cols]
    return m, x.double() * s


def columns(m, to):
    return api.Quantized(m.q[:, :to], m.scales[:, :-(-to // 128)], m.block)


# few rows; tiles in one, two and four groups of wavefronts; split; 256x256 (bf16, both)
@pytest.mark.parametrize("m,n", [(1, 40), (3, 5000), (30, 64), (40, 100), (300, 260), (700, 900), (1000, 1000), (2100, 8000), (4000, 4200)])
@pytest.mark.parametrize("k", [1, 7, 15, 17, 120, 130, 300, 1001])
def test_what_lies_past_the_last_column_is_not_read_as_values(m, n, k):
    """Sums of integers below 2^16 by halves: exact in either form.  0x7F is a NaN, 0x7E is 448."""
    for past, other in ((0x7F, 0x7F), (0x7E, 0xFE), (0x7F, 0), (0, 0xFF)):
        (a, a64), (b, b64) = integers(m, k, 1, m + k, past), integers(n, k, 128, n + k, other)
        ref = a64 @ b64.t().contiguous()
        assert torch.equal(api.product(a, b, dtype=api.F32).double(), ref)
        assert torch.equal(api.product(a, b).double(), ref.to(torch.bfloat16).double())
        if m * n > 1 << 22:
            break


@pytest.mark.parametrize("m,n", [(2, 64), (50, 70), (300, 500), (4000, 4200)])
def test_the_first_columns_of_a_wider_matrix(m, n):
    (a, a64), (b, b64) = integers(m, 700, 1, 1, 0x7F), integers(n, 700, 128, 2, 0x7F)
    for k in (5, 100, 128, 300, 511, 640, 699):
        ref = a64[:, :k].contiguous() @ b64[:, :k].t().contiguous()
        assert torch.equal(api.product(columns(a, k), columns(b, k), dtype=api.F32).double(), ref)
        assert torch.equal(api.product(columns(a, k), columns(b, k)).double(), ref.to(torch.bfloat16).double())


@pytest.mark.parametrize("m,n,k", [(64, 64, 16300), (100, 500, 6199), (130, 2000, 7001), (714, 174, 1399), (1000, 512, 907)])
def test_what_lies_past_a_long_contraction(m, n, k):
    (a, a64), (b, b64) = integers(m, k, 1, m, 0x7F), integers(n, k, 1, n, 0x7F)
    ref = a64 @ b64.t().contiguous()
    assert torch.equal(api.product(a, b, dtype=api.F32).double(), ref)
    assert torch.equal(api.product(a, b, dtype=api.F32, out=torch.empty(m, n + 5, device=DEV)[:, 2:n + 2]).double(), ref)


SHAPES = [(1, 40), (3, 5000), (30, 64), (40, 100), (300, 260), (1000, 1000), (4000, 4200)]


@pytest.mark.parametrize("m,n", SHAPES)
@pytest.mark.parametrize("ea,eb", [(246, 10), (10, 246), (227, 27), (27, 227), (127, 127)])
def test_scales_far_apart(m, n, ea, eb):
    """Values at 2^119 and 2^-117, between which both forms are exact: their products are integers."""
    for k in (90, 400):
        (a, a64), (b, b64) = integers(m, k, 1, m, 0x7F), integers(n, k, 128, n, 0x7F)
        a64, b64 = a.q.float().double(), b.q.float().double()
        a.scales.view(torch.uint8).fill_(ea)
        b.scales.view(torch.uint8).fill_(eb)
        ref = a64 @ b64.t().contiguous() * 2.0 ** (ea + eb - 254)
        assert torch.equal(api.product(a, b, dtype=api.F32).double(), ref)
        assert torch.equal(api.product(a, b).double(), ref.to(torch.bfloat16).double())
        assert torch.equal(api.product(a, b, float32_sums=True).double(), ref.to(torch.bfloat16).double())


@pytest.mark.parametrize("m,n", SHAPES)
@pytest.mark.parametrize("k", [100, 400])
def test_what_is_not_finite_stays_in_its_row_and_block_in_both_forms(m, n, k):
    g = torch.Generator(device=DEV)
    g.manual_seed(m)
    x, w = torch.randn(m, k, device=DEV, generator=g), torch.randn(n, k, device=DEV, generator=g)
    x[m // 2, k - 1] = float("inf")
    w[n - 1, 3] = float("nan")                   # a block of up to 128 rows of weights
    x8, w8, first = api.quantize(x).rows, api.quantize(w, block=128).rows, (n - 1) // 128 * 128
    for dtype, sums in ((api.F32, False), (api.BF16, False), (api.BF16, True)):
        for relu in (False, True):
            bad = api.product(x8, w8, dtype=dtype, float32_sums=sums, relu=relu).isnan()
            assert bool(bad[m // 2].all()) and bool(bad[:, first:].all())
            bad[m // 2] = False
            assert not bool(bad[:, :first].any())


@pytest.mark.parametrize("m,n,k", [(4000, 4200, 300), (4093, 4099, 277), (3111, 5003, 1291)])
def test_large_ragged_products_into_a_wider_matrix(m, n, k):
    (a, a64), (b, b64) = integers(m, k, 1, m, 0), integers(n, k, 128, n, 0)
    bias = torch.arange(n, device=DEV).float() % 7 - 3
    ref = (a64 @ b64.t().contiguous() + bias.double()).clamp(min=0)
    for dtype in (torch.float32, torch.bfloat16):
        room = torch.full((m + 2, n + 9), 7.0, dtype=dtype, device=DEV)
        for first in (0, 1, 8):
            api.product(a, b, bias=bias, relu=True, out=room[1:m + 1, first:first + n])
            assert torch.equal(room[1:m + 1, first:first + n].double(), ref.to(dtype).double())
            room[1:m + 1, first:first + n] = 7.0
            assert bool((room == 7.0).all())


def test_shapes_and_sums_of_empty_matrices():
    for shape in ((0, 5), (5, 0), (0, 0)):
        r = api.quantize(torch.empty(shape, device=DEV), transposed=True, column_sums=True)
        assert tuple(r.rows.q.shape) == shape and tuple(r.transposed.q.shape) == shape[::-1]
        assert r.column_sums.tolist() == [0.0] * shape[1]
