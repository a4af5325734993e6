"""The 8-bit operators and gradient clipping on the GPU against the float64 oracle.

Tolerances, with u = 2^-24 (rounding to the 24 bits of float32) and 2^-8 (to the 8 of bf16):
  quantising     exact: the largest magnitude, the power of two and the rounding are
  product        a sum of K exact products in float32 in any order is within (K + 2) u of the sum of their magnitudes, bias and rounding
                 included; a bf16 output adds 2^-8 of its value.  On small integers every partial sum is exact, and so must the output be
  norm           the sum of squares is added in at most 40 steps a lane, 10 across, then 5 roundings: 64 u of rstd, 70 u of y;
                 the 8-bit values are the nearest to something within that of the oracle's
  its backward   64 u of the sum of the magnitudes of dx's terms; (rows + 8) u of dgamma's
  clipping       the norm 2 u (float64 sums, rounded once), the values 3 u, and 2^-149 where they leave float32's range
"""

import ctypes

import numpy as np
import pytest
import torch

from oracle import eightbit as o8
from paper_2403_11204_amd import api

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def values(shape, seed, dtype=torch.float32, spread=1.0):
    g = np.random.default_rng(seed)
    x = g.normal(0, 1, shape) * np.exp(spread * g.normal(0, 1, (shape[0],) + (1,) * (len(shape) - 1)))
    return torch.from_numpy(x.astype(np.float32)).to(dtype)


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def bytes_of(t):
    return t.cpu().contiguous().view(torch.uint8).numpy()


def pads_are_zero(m):
    """The bytes from the last column up to the next 16 are zero."""
    rows, cols = m.q.shape
    ld = m.q.stride(0)
    full = m.q.view(torch.uint8).as_strided((rows, -(-cols // 16) * 16), (ld, 1)).cpu().numpy()
    return not full[:, cols:].any()


def check_quantized(m, x64, block):
    q, e = o8.quantize(x64, block)
    assert np.array_equal(bytes_of(m.scales), (e + 127).astype(np.uint8))
    assert np.array_equal(bytes_of(m.q), o8.bits_of(np.where(q == 0, np.copysign(0.0, x64), q)))
    assert pads_are_zero(m)


def eight(x, block):
    """A float64 matrix as an 8-bit one on the GPU (by the oracle), and the float64 matrix that it stands for."""
    q, e = o8.quantize(x, block)
    m = api.empty_quantized(*x.shape, block)
    m.q.view(torch.uint8).as_strided((x.shape[0], m.q.stride(0)), (m.q.stride(0), 1)).zero_()
    m.q.view(torch.uint8).copy_(torch.from_numpy(o8.bits_of(q)))
    m.scales.view(torch.uint8).copy_(torch.from_numpy((e + 127).astype(np.uint8)))
    return m, o8.dequantize(q, e, block)


# ---- quantising ---------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 784), (5, 127), (128, 128), (129, 16), (47, 129), (200, 1000), (333, 513), (300, 2052)])
def test_quantize(rows, cols, block, dtype):
    x = values((rows, cols), rows * cols, TYPES[dtype], 3.0)
    x[rows // 2, : cols // 2] = 0
    r = api.quantize(x.to(DEV), block=block, transposed=True)
    check_quantized(r.rows, f64(x), block)
    check_quantized(r.transposed, f64(x).T, block)
    assert r.column_sums is None
    one = api.quantize(x.to(DEV), block=block)
    assert one.transposed is None and np.array_equal(bytes_of(one.rows.q), bytes_of(r.rows.q)) and np.array_equal(bytes_of(one.rows.scales), bytes_of(r.rows.scales))
    assert pads_are_zero(one.rows)
    other = api.quantize(x.to(DEV), block=block, rows=False, transposed=True)
    assert other.rows is None and np.array_equal(bytes_of(other.transposed.q), bytes_of(r.transposed.q))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 40), (130, 260), (1410, 60), (513, 2049)])
def test_quantize_with_mask_and_sums(rows, cols, dtype):
    x, a = values((rows, cols), 7, TYPES[dtype]), values((rows, cols), 8, TYPES[dtype]).clamp(min=0)
    a[:, 3] = 0                                  # a column and a row that pass nothing
    a[rows - 1] = 0
    a[0, 5] = -1.0
    kept = np.where(f64(a) > 0, f64(x), 0.0)
    r = api.quantize(x.to(DEV), transposed=True, mask=a.to(DEV), column_sums=True)
    check_quantized(r.rows, np.where(f64(a) > 0, f64(x), 0.0), 1)
    check_quantized(r.transposed, kept.T, 1)
    assert np.all(np.abs(f64(r.column_sums) - kept.sum(0)) <= (rows + 2) * U * np.abs(kept).sum(0))
    alone = api.quantize(x.to(DEV), mask=a.to(DEV))
    assert np.array_equal(bytes_of(alone.rows.q), bytes_of(r.rows.q))
    sums = api.quantize(x.to(DEV), mask=a.to(DEV), column_sums=True)
    assert torch.equal(sums.column_sums, r.column_sums) and np.array_equal(bytes_of(sums.rows.q), bytes_of(r.rows.q))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_quantize_at_any_offset_and_stride(dtype):
    big = values((70, 700), 3, TYPES[dtype])
    for off, cols in ((0, 256), (1, 256), (3, 131), (7, 640)):
        x = big.to(DEV)[2:60, off:off + cols]
        r = api.quantize(x, transposed=True)
        check_quantized(r.rows, f64(big)[2:60, off:off + cols], 1)
        check_quantized(r.transposed, f64(big)[2:60, off:off + cols].T, 1)


def test_quantize_what_is_tiny_huge_or_not_finite():
    x = torch.zeros(6, 256)
    x[0, 0], x[0, 130] = 1e-45, 448.0
    x[1, 5], x[1, 200] = 3.4e38, float(np.nextafter(np.float32(448), np.float32(500)))
    x[2, 5] = float("inf")
    x[3, 250] = float("nan")
    x[4, 1] = -float("inf")
    x[5, 0] = 2.0 ** -127
    r = api.quantize(x.to(DEV), transposed=True)
    fine = [0, 1, 5]
    q, e = o8.quantize(f64(x)[fine], 1)
    assert np.array_equal(bytes_of(r.rows.scales)[fine], (e + 127).astype(np.uint8)) and np.array_equal(f64(r.rows.q)[fine], q)
    s = bytes_of(r.rows.scales)
    assert s[2, 0] == 255 and s[2, 1] == 0 and s[3, 0] == 0 and s[3, 1] == 255 and s[4, 0] == 255
    assert bytes_of(r.transposed.scales)[[5, 250, 1, 6], 0].tolist() == [255, 255, 255, 0]
    assert np.all(bytes_of(api.quantize(x.to(DEV), block=128).rows.scales) == 255)


def test_empty_matrices():
    for shape in ((0, 5), (5, 0), (0, 0)):
        r = api.quantize(torch.empty(shape, device=DEV), transposed=True, column_sums=True)
        assert tuple(r.rows.q.shape) == shape and f64(r.column_sums).tolist() == [0.0] * shape[1] or shape[0]
    n = api.rmsnorm(torch.empty(0, 16, device=DEV))
    assert n.rstd.numel() == 0
    dx, dgamma = api.rmsnorm_backward(*[torch.empty(0, 16, device=DEV)] * 2, None, torch.empty(0, device=DEV))
    assert dx.shape == (0, 16) and not f64(dgamma).any()
    k0 = api.product(api.empty_quantized(3, 0), api.empty_quantized(4, 0), bias=torch.tensor([1.0, -2.0, 3.0, 0.0], device=DEV), relu=True, dtype=api.F32)
    assert np.array_equal(f64(k0), np.tile([1.0, 0.0, 3.0, 0.0], (3, 1)))
    assert api.product(api.empty_quantized(0, 20), api.empty_quantized(4, 20)).shape == (0, 4)


# ---- products -----------------------------------------------------------------------------------------------------
SHAPES = [(1, 1, 1), (1, 16, 16), (1, 47, 60), (1, 1000, 784), (2, 64, 128), (3, 65, 129), (5, 200, 3001), (8, 130, 640), (15, 129, 1500), (16, 512, 2048), (17, 96, 400),
          (33, 100, 1000), (64, 64, 64), (64, 333, 4100), (100, 129, 777), (130, 260, 131), (256, 512, 1024), (300, 700, 1500), (1000, 777, 300), (1410, 80, 784), (130, 2000, 131), (70, 300, 9000), (2000, 2100, 200), (2000, 4090, 600),
          (4100, 4200, 144), (4096, 4096, 3200)]


@pytest.mark.parametrize("m,n,k", SHAPES)
def test_product_of_small_integers_is_exact(m, n, k):
    """Values of -2 .. 2 at scales of 2^-2 .. 2^1: every sum of products is a multiple of 2^-4 below 2^20, exact in float32."""
    g = torch.Generator(device=DEV)
    g.manual_seed(m + 3 * n + 7 * k)

    def made(rows, block):
        full = api.empty_quantized(rows, k, block)
        ints = torch.randint(-2, 3, (rows, k), device=DEV, generator=g).float()
        full.q.view(torch.uint8).as_strided((rows, full.q.stride(0)), (full.q.stride(0), 1)).zero_()
        full.q.copy_(ints.to(torch.float8_e4m3fn))
        e = torch.randint(125, 129, full.scales.shape, device=DEV, generator=g)
        full.scales.view(torch.uint8).copy_(e.to(torch.uint8))
        s = torch.exp2((e - 127).double()).repeat_interleave(block, 0)[:rows].repeat_interleave(128, 1)[:, :k]
        return full, ints.double() * s

    (a, a64), (b, b64), (c, c64) = made(m, 1), made(n, 128), made(n, 1)
    bias = torch.randint(-3, 4, (n,), device=DEV, generator=g).float()
    ref = a64 @ b64.t().contiguous()
    assert torch.equal(api.product(a, b, dtype=api.F32).double(), ref)
    assert torch.equal(api.product(a, b, bias=bias, relu=True, dtype=api.F32).double(), (ref + bias.double()).clamp(min=0))
    ref = a64 @ c64.t().contiguous()
    assert torch.equal(api.product(a, c, bias=bias).double(), (ref + bias.double()).to(torch.bfloat16).double())
    assert torch.equal(api.product(c, a, dtype=api.F32).double(), ref.t())
    if n >= 128:
        assert torch.equal(api.product(b, a, dtype=api.F32).double(), (a64 @ b64.t().contiguous()).t())      # blocks on the left


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(1, 300, 784), (4, 96, 4100), (16, 130, 1000), (40, 260, 900), (333, 300, 1000), (300, 260, 2500)])
def test_product_of_quantized_values(m, n, k, dtype):
    (a, a64), (b, b64) = eight(f64(values((m, k), 1)), 1), eight(f64(values((n, k), 2)), 128)
    bias = values((n,), 3, spread=0.0)
    ref = o8.product(a64, b64, f64(bias), relu=True)
    got = f64(api.product(a, b, bias=bias.to(DEV), relu=True, dtype=api.BF16 if dtype == "bf16" else api.F32))
    size = np.abs(a64) @ np.abs(b64).T + np.abs(f64(bias))
    assert np.all(np.abs(got - ref) <= (k + 2) * U * size + (2.0 ** -8 * np.abs(ref) if dtype == "bf16" else 0))


def test_product_into_a_strided_output_leaves_the_rest():
    (a, a64), (b, b64) = eight(f64(values((30, 200), 1)), 1), eight(f64(values((101, 200), 2)), 128)
    for dtype in (torch.float32, torch.bfloat16):
        for first in (0, 1, 5):
            room = torch.full((32, 120), 7.0, dtype=dtype, device=DEV)
            api.product(a, b, out=room[1:31, first:first + 101])
            whole = f64(room)
            ref = a64 @ b64.T
            assert np.all(np.abs(whole[1:31, first:first + 101] - ref) <= 202 * U * (np.abs(a64) @ np.abs(b64).T) + 2.0 ** -8 * np.abs(ref))
            whole[1:31, first:first + 101] = 7.0
            assert np.all(whole == 7.0)


@pytest.mark.parametrize("m", [3, 40, 300])
def test_what_is_not_finite_stays_in_its_row(m):
    x = values((m, 400), 5)
    x[1, 300] = float("inf")
    a = api.quantize(x.to(DEV)).rows
    b, b64 = eight(f64(values((70, 400), 6)), 128)
    got = f64(api.product(a, b, relu=True, dtype=api.F32))
    assert np.all(np.isnan(got[1])) and np.all(np.isfinite(np.delete(got, 1, 0)))
    tiny = torch.full((m, 400), 1e-42)                   # scales of 2^-127: products underflow, nothing else happens
    assert np.all(np.abs(f64(api.product(api.quantize(tiny.to(DEV)).rows, b, dtype=api.F32))) < 1e-38)


def test_product_of_a_matrix_past_four_gigabytes():
    rows, k = 270000, 16384
    a = api.empty_quantized(rows, k)
    assert rows * a.q.stride(0) > 1 << 32
    a.q.view(torch.uint8).fill_(0)
    a.scales.view(torch.uint8).fill_(127)
    pick = [0, 1, 131071, 131072, 200001, rows - 1]
    x = torch.randint(-4, 5, (len(pick), k), device=DEV).float()
    a.q[pick] = x.to(torch.float8_e4m3fn)
    b = api.quantize(torch.randint(-4, 5, (20, k), device=DEV).float(), block=128).rows
    ref = x.double() @ _dequantized(b).t().contiguous()
    out = api.product(a, b, dtype=api.F32)
    assert torch.equal(out[pick].double(), ref)
    out[pick] = 0
    assert not out.any()


def _dequantized(m):
    rows, cols = m.q.shape
    s = m.scales.float().double().repeat_interleave(m.block, 0)[:rows].repeat_interleave(128, 1)[:, :cols]
    return m.q.float().double() * s


# ---- the norm -----------------------------------------------------------------------------------------------------
DIMS = [(1, 1), (1, 4096), (3, 7), (5, 128), (7, 129), (9, 512), (6, 513), (33, 777), (5, 1024), (5, 1030), (4, 2048), (4, 3001), (4, 4096), (3, 5000), (3, 8192), (2, 16000),
        (2, 16384), (2, 16392), (2, 20001), (300, 64)]


def check_norm(n, x, r, gamma, eps, dtype):
    total = f64(x) if r is None else f64((x.float() + r.float()).to(dtype))
    assert np.array_equal(f64(n.h), total)
    y, rstd = o8.rmsnorm(total, f64(gamma)[None], eps)
    assert np.all(np.abs(f64(n.rstd) - rstd) <= 64 * U * rstd)
    close = 70 * U * np.abs(y)
    if n.y is not None:
        assert np.all(np.abs(f64(n.y) - y) <= close + (2.0 ** -8 * np.abs(y) if dtype is torch.bfloat16 else 0))
    e = o8.exponents(y, 1)
    got = bytes_of(n.y8.scales).astype(np.int64) - 127
    for i, j in np.argwhere(got != e):                # only where the largest value is that close to the line between two scales
        big = np.abs(y[i, j * 128:(j + 1) * 128]).max()
        assert abs(got[i, j] - e[i, j]) == 1 and min(abs(big / (448 * 2.0 ** k) - 1) for k in (e[i, j], e[i, j] - 1)) <= 70 * U
    s = 2.0 ** o8.spread(got, 1, y.shape)
    step = np.maximum(2.0 ** np.floor(np.log2(np.maximum(np.abs(y / s), 2.0 ** -6))), 2.0 ** -6) / 8 * s
    assert np.all(np.abs(f64(n.y8.q) * s - y) <= step / 2 + close)
    assert pads_are_zero(n.y8)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,dim", DIMS)
def test_rmsnorm(rows, dim, dtype):
    dt = TYPES[dtype]
    x, r, gamma = values((rows, dim), dim, dt), values((rows, dim), dim + 1, dt), 1 + 0.1 * values((dim,), 5, spread=0.0)
    check_norm(api.rmsnorm(x.to(DEV), gamma.to(DEV), residual=r.to(DEV), eps=1e-5, normed=True), x, r, gamma, 1e-5, dt)
    check_norm(api.rmsnorm(x.to(DEV), gamma.to(DEV), eps=1e-6), x, None, gamma, 1e-6, dt)
    plain = api.rmsnorm(x.to(DEV), normed=True, quantized=False)
    assert plain.y8 is None
    y = o8.rmsnorm(f64(x), np.ones((1, dim)), 1e-6)[0]
    assert np.all(np.abs(f64(plain.y) - y) <= (70 * U + (2.0 ** -8 if dtype == "bf16" else 0)) * np.abs(y))


def test_rmsnorm_of_views_of_nothing_and_of_what_is_not_finite():
    big, r = values((40, 900), 1, torch.bfloat16), values((40, 777), 2, torch.bfloat16)
    gamma = torch.ones(777)
    view = big.to(DEV)[3:36, 5:782]
    check_norm(api.rmsnorm(view, gamma.to(DEV), residual=r.to(DEV)[3:36]), big[3:36, 5:782], r[3:36], gamma, 1e-6, torch.bfloat16)
    x = torch.zeros(3, 256)
    x[1, 7], x[2] = float("inf"), 1e-30
    n = api.rmsnorm(x.to(DEV), eps=1e-6, normed=True)
    y = f64(n.y)
    assert not y[0].any() and abs(f64(n.rstd)[0] - 1000) <= 64 * U * 1000 and not f64(n.y8.q)[0].any()
    assert np.isnan(y[1, 7]) and f64(n.rstd)[1] == 0 and bytes_of(n.y8.scales)[1].tolist() == [255, 0]
    assert np.all(np.abs(y[2] / 1e-27 - 1) < 1e-6)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,dim", DIMS + [(1000, 300), (513, 2050), (700, 4096)])
def test_rmsnorm_backward(rows, dim, dtype):
    dt = TYPES[dtype]
    h, dy, dh, gamma = values((rows, dim), 1, dt), values((rows, dim), 2, dt), values((rows, dim), 3, dt), 1 + 0.1 * values((dim,), 5, spread=0.0)
    rstd = torch.from_numpy((1 / np.sqrt(np.mean(f64(h) ** 2, 1) + 1e-6)).astype(np.float32))
    n, y, x, g = f64(rstd)[:, None], f64(dy), f64(h), f64(gamma)[None]
    for past in (dh, None):
        dx, dgamma = api.rmsnorm_backward(dy.to(DEV), h.to(DEV), gamma.to(DEV), rstd.to(DEV), dh=past.to(DEV) if past is not None else None)
        extra = f64(past) if past is not None else np.zeros_like(x)
        ref = extra + n * (g * y - x * n * n * np.mean(g * y * x, 1, keepdims=True))
        size = np.abs(extra) + n * (np.abs(g * y) + np.abs(x) * n * n * np.mean(np.abs(g * y * x), 1, keepdims=True))
        assert np.all(np.abs(f64(dx) - ref) <= 64 * U * size + (2.0 ** -8 * np.abs(ref) if dtype == "bf16" else 0))
        assert np.all(np.abs(f64(dgamma) - (y * x * n).sum(0)) <= (rows + 8) * U * np.abs(y * x * n).sum(0))
    ones, none = api.rmsnorm_backward(dy.to(DEV), h.to(DEV), None, rstd.to(DEV), gamma_grad=False)
    assert none is None
    ref = n * (y - x * n * n * np.mean(y * x, 1, keepdims=True))
    size = n * (np.abs(y) + np.abs(x) * n * n * np.mean(np.abs(y * x), 1, keepdims=True))
    assert np.all(np.abs(f64(ones) - ref) <= 64 * U * size + (2.0 ** -8 * np.abs(ref) if dtype == "bf16" else 0))


@pytest.mark.parametrize("rows,dim", [(9, 300), (40, 4096), (3, 20001)])
def test_rmsnorm_and_its_backward_in_place(rows, dim):
    L, st = api.lib(), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    x, r, dy = (values((rows, dim), i, torch.bfloat16).to(DEV) for i in range(3))
    gamma = torch.ones(dim, device=DEV)
    ref = api.rmsnorm(x, gamma, residual=r, normed=True)
    h = r.clone()
    y, rstd = torch.empty_like(x), torch.empty(rows, device=DEV)
    assert L.slp_rmsnorm(api._ptr(x), dim, api._ptr(h), dim, api._ptr(gamma), 1e-6, api.BF16, rows, dim, api._ptr(h), dim, api._ptr(y), dim, None, 0, None, 0,
                         api._ptr(rstd), st) == 0
    assert torch.equal(h, ref.h) and torch.equal(y, ref.y) and torch.equal(rstd, ref.rstd)
    dx, dgamma = api.rmsnorm_backward(dy, h, gamma, rstd, dh=x)
    size = L.slp_rmsnorm_backward_workspace_bytes(rows, dim)
    work, dg = torch.empty(size, dtype=torch.uint8, device=DEV), torch.empty(dim, device=DEV)
    for into in (dy.clone(), x.clone()):
        a, b = (into, x) if torch.equal(into, dy) else (dy, into)
        assert L.slp_rmsnorm_backward(api._ptr(a), dim, api._ptr(h), dim, api._ptr(gamma), api._ptr(rstd), api._ptr(b), dim, api.BF16, rows, dim, api._ptr(into), dim,
                                      api._ptr(dg), api._ptr(work), size, st) == 0
        assert torch.equal(into, dx) and torch.equal(dg, dgamma)


# ---- clipping -----------------------------------------------------------------------------------------------------
def check_clip(tensors, max_norm):
    ref_norm, ref = o8.clip([f64(t) for t in tensors], max_norm)
    on = [t.to(DEV) for t in tensors]
    out = [torch.full_like(t, 9.0) for t in on]
    norm = api.clip_gradients(on, max_norm, out=out)
    assert abs(float(norm) - ref_norm) <= 2 * U * ref_norm and float(api.gradient_norm(on)) == float(norm)
    for t, o, r, before in zip(on, out, ref, tensors):
        half = 2.0 ** -8 if t.dtype is torch.bfloat16 else 0
        assert np.all(np.abs(f64(o) - r) <= (3 * U + half) * np.abs(r) + 2.0 ** -149) and torch.equal(t.cpu(), before)
    assert float(api.clip_gradients(on, max_norm)) == float(norm)
    assert all(torch.equal(t, o) for t, o in zip(on, out))


@pytest.mark.parametrize("share", [0.3, 5.0])
@pytest.mark.parametrize("sizes", [[1], [7], [8192], [8193, 1, 0, 5], [100000, 3, 70001], [1 + i % 5 for i in range(130)], [3000000]])
def test_clip(sizes, share):
    tensors = [values((n,), i, [torch.float32, torch.bfloat16][i % 2], 0.0) if n else torch.empty(0) for i, n in enumerate(sizes)]
    check_clip(tensors, share * float(np.sqrt(sum(sizes))))


def test_clip_keeps_its_range_and_leaves_what_is_not_finite():
    check_clip([torch.tensor([1e30, -3e37, 1e-30])], 2.0)
    check_clip([torch.tensor([1e-30, 2e-38])], 1e-31)
    for bad in (float("inf"), float("nan")):
        t = torch.tensor([1.0, bad, 2.0]), torch.arange(5.0)
        on = [x.to(DEV) for x in t]
        norm = api.clip_gradients(on, 0.5)
        assert not np.isfinite(float(norm)) and torch.equal(on[1].cpu(), t[1]) and float(on[0][0]) == 1.0
    zero = torch.zeros(10, device=DEV)
    assert float(api.clip_gradients([zero], 1.0)) == 0.0 and not zero.any()


def test_clip_of_views_at_any_element():
    room = torch.arange(40.0, device=DEV)
    half = room.to(torch.bfloat16)
    assert abs(float(api.gradient_norm([room[1:20], half[3:10]])) - np.sqrt(sum(i * i for i in range(1, 20)) + sum(i * i for i in range(3, 10)))) < 1e-4
    api.clip_gradients([room[1:20]], 1.0)
    assert float(room[0]) == 0.0 and float(room[20]) == 20.0 and abs(float(room[1:20].norm()) - 1) < 1e-5


# ---- streams, repetition, graphs ----------------------------------------------------------------------------------
def everything(x, r, gamma, w, dy):
    n = api.rmsnorm(x, gamma, residual=r, normed=True)
    w8 = api.quantize(w, block=128, transposed=True)
    z = api.product(n.y8, w8.rows, relu=True, dtype=api.F32)
    dz = api.quantize(dy, transposed=True, mask=z, column_sums=True)
    yt = api.quantize(n.y, rows=False, transposed=True).transposed
    dyn = api.product(dz.rows, w8.transposed, dtype=api.F32)
    dw = api.product(dz.transposed, yt, dtype=api.F32)
    dx, dgamma = api.rmsnorm_backward(dyn, n.h, gamma, n.rstd, dh=dyn)
    grads = [dw, dz.column_sums, dgamma]
    out = [torch.empty_like(g) for g in grads]
    norm = api.clip_gradients(grads, 0.01, out=out)
    return [z, dx, norm] + out


def test_another_stream_repetition_and_capture():
    x, r, gamma, w, dy = values((70, 300), 1).to(DEV), values((70, 300), 2).to(DEV), torch.ones(300, device=DEV), values((200, 300), 3).to(DEV), values((70, 200), 4).to(DEV)
    ref = [t.clone() for t in everything(x, r, gamma, w, dy)]
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(everything(x, r, gamma, w, dy), ref))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = everything(x, r, gamma, w, dy)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(other, ref))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = everything(x, r, gamma, w, dy)
    for k in range(3):
        x.copy_(values((70, 300), 10 + k).to(DEV))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        assert all(torch.equal(a, b) for a, b in zip(got, everything(x, r, gamma, w, dy)))


# ---- outputs of a few columns for many rows, and contractions of nothing ----------------------------------------------
@pytest.mark.parametrize("m,n", [(37000, 10), (37000, 100), (37000, 128), (37000, 129), (10, 37000)])
def test_narrow_products_of_many_rows(m, n):
    k = 300
    a = api.quantize(torch.randint(-4, 5, (m, k), device=DEV).float()).rows
    b = api.quantize(torch.randint(-4, 5, (n, k), device=DEV).float(), block=128).rows
    ref = _dequantized(a) @ _dequantized(b).t().contiguous()         # integers below 2^13
    assert torch.equal(api.product(a, b, dtype=api.F32).double(), ref)
    assert torch.equal(api.product(a, b).double(), ref.to(torch.bfloat16).double())


@pytest.mark.parametrize("m,n", [(3, 40), (300, 40), (100, 2000)])
def test_a_contraction_of_nothing_reads_nothing_whatever_its_leading_dimensions(m, n):
    out = torch.full((m, n), 7.0, device=DEV)
    bias = torch.arange(n, device=DEV).float()
    need = api.lib().slp_product_workspace_bytes(m, n, 0)
    assert need == 0
    rc = api.lib().slp_product(None, -31, None, -7, 1, None, -(1 << 33), None, 5, 128, bias.data_ptr(), 0, m, n, 0, out.data_ptr(), n, api.F32, None, 0, api._stream())
    assert rc == 0 and torch.equal(out, bias.expand(m, n))


@pytest.mark.parametrize("m,n,k", [(714, 174, 1400), (300, 300, 1409), (65, 65, 3000), (1000, 512, 900), (1000, 500, 5000), (700, 900, 1025), (1000, 1000, 4000), (1200, 1100, 2050),
                                   (64, 64, 16384), (100, 500, 6200), (130, 2000, 7000), (10, 1000, 20001)])
def test_contractions_shared_by_groups_of_wavefronts_and_workgroups(m, n, k):
    """Integers: the parts' sums are exact whatever the order; the same call gives the same bits."""
    g = torch.Generator(device=DEV)
    g.manual_seed(k)
    a = api.quantize(torch.randint(-4, 5, (m, k), device=DEV, generator=g).float()).rows
    b = api.quantize(torch.randint(-4, 5, (n, k), device=DEV, generator=g).float(), block=128).rows
    bias = torch.randint(-9, 10, (n,), device=DEV, generator=g).float()
    ref = _dequantized(a) @ _dequantized(b).t().contiguous()
    assert torch.equal(api.product(a, b, dtype=api.F32).double(), ref)
    assert torch.equal(api.product(a, b, bias=bias, relu=True).double(), (ref + bias).clamp(min=0).to(torch.bfloat16).double())
    x, y = values((m, k), 3).to(DEV), values((n, k), 4).to(DEV)
    x, y = api.quantize(x).rows, api.quantize(y).rows
    for dtype in (api.F32, api.BF16):
        assert torch.equal(api.product(x, y, dtype=dtype), api.product(x, y, dtype=dtype))


def test_outputs_of_a_small_call_lie_apart_and_outlive_one_another():
    x, r = (values((3, 200), i, torch.bfloat16).to(DEV) for i in range(2))
    gamma = torch.ones(200, device=DEV)

    def outputs():
        n = api.rmsnorm(x, gamma, residual=r, normed=True)
        q = api.quantize(x, transposed=True, mask=r, column_sums=True)
        dx, dgamma = api.rmsnorm_backward(x, n.h, gamma, n.rstd)
        return [n.h, n.rstd, n.y, n.y8.q, n.y8.scales, q.rows.q, q.rows.scales, q.transposed.q, q.transposed.scales, q.column_sums, dx, dgamma, api.gradient_norm([x, r])]

    first = outputs()
    spans = sorted((t.data_ptr(), t.data_ptr() + (t.numel() and 1 + sum((s - 1) * st for s, st in zip(t.shape, t.stride()))) * t.element_size()) for t in first)
    assert all(a[1] <= b[0] for a, b in zip(spans, spans[1:]))
    assert all(t.data_ptr() % 256 == 0 for t in first)
    kept = [f64(t) if t.dtype != torch.float8_e8m0fnu else bytes_of(t).copy() for t in first]
    h = first[0]
    del first
    for _ in range(50):
        again = outputs()
        for t in again:
            t.view(torch.uint8).fill_(85) if t.is_contiguous() and t.dim() else None
    assert np.array_equal(f64(h), kept[0])
    for t, k in zip(outputs(), kept):
        assert np.array_equal(f64(t) if t.dtype != torch.float8_e8m0fnu else bytes_of(t), k)


@pytest.mark.parametrize("rows,dim", [(1, 16384), (1, 1025), (4, 1000), (2, 60), (5, 1000), (2, 4096)])
def test_rmsnorm_backward_of_few_rows(rows, dim):
    h, dy = values((rows, dim), 1), values((rows, dim), 2)
    n = api.rmsnorm(h.to(DEV), quantized=False)
    dx, dgamma = api.rmsnorm_backward(dy.to(DEV), h.to(DEV), None, n.rstd)
    terms = f64(dy) * f64(h) * f64(n.rstd)[:, None]
    assert np.all(np.abs(f64(dgamma) - terms.sum(0)) <= (rows + 4) * U * np.abs(terms).sum(0))
    assert api.rmsnorm_backward(dy.to(DEV), h.to(DEV), None, n.rstd, gamma_grad=False)[1] is None


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,dim", [(1100, 1500), (4100, 1030), (600, 9001), (3, 12288), (520, 12289), (2, 13000), (33000, 24), (9000, 100), (4100, 200), (17, 256),
                                      (4099, 257)])
def test_rmsnorm_where_workgroups_take_several_rows(rows, dim, dtype):
    test_rmsnorm(rows, dim, dtype)
    test_rmsnorm_backward(rows, dim, dtype)


@pytest.mark.parametrize("m,n,k", [(581, 14917, 256), (581, 14914, 130), (2050, 8200, 200), (247, 1024, 8192), (200, 400, 12000), (1000, 512, 6200), (7759, 234, 4100)])
def test_products_at_the_borders_of_the_rules(m, n, k):
    g = torch.Generator(device=DEV)
    g.manual_seed(n)
    a = api.quantize(torch.randint(-4, 5, (m, k), device=DEV, generator=g).float()).rows
    b = api.quantize(torch.randint(-4, 5, (n, k), device=DEV, generator=g).float(), block=128).rows
    ref = _dequantized(a) @ _dequantized(b).t().contiguous()
    assert torch.equal(api.product(a, b, dtype=api.F32).double(), ref)
    assert torch.equal(api.product(a, b).double(), ref.to(torch.bfloat16).double())
    room = torch.full((m, n + 3), 7.0, dtype=torch.bfloat16, device=DEV)
    api.product(a, b, out=room[:, 1:n + 1])
    assert torch.equal(room[:, 1:n + 1].double(), ref.to(torch.bfloat16).double()) and bool((room[:, 0] == 7).all()) and bool((room[:, n + 1:] == 7).all())
