"""What the 8-bit operators and gradient clipping refuse, before any device is touched.  CPU only."""

import ctypes

import pytest

from paper_2403_11204_amd import api

P = 0x100000          # an address that is never followed
ARG, SHAPE, ALLOC = -1, -2, -3


def refused(code, got, word=None):
    assert got == code, (got, api.lib().slp_last_error())
    if word:
        assert word in api.lib().slp_last_error(), api.lib().slp_last_error()


def quantize(**kw):
    a = dict(x=P, ldx=300, mask=None, ldmask=0, dt=0, rows=10, cols=300, block=1, q=P, ldq=384, scales=P, lds=4, qt=None, ldqt=0, scales_t=None, ldst=0,
             sums=None, work=None, size=0)
    a.update(kw)
    return api.lib().slp_quantize(*a.values(), None)


def test_quantize():
    refused(ARG, quantize(x=None), b"null")
    refused(ARG, quantize(dt=2), b"dtype")
    refused(ARG, quantize(block=64), b"blocks")
    refused(ARG, quantize(rows=-1), b"negative")
    refused(ARG, quantize(q=None, scales=None), b"no output")
    refused(ARG, quantize(scales=None), b"scales")
    refused(ARG, quantize(qt=P, ldqt=16), b"scales")
    refused(SHAPE, quantize(ldx=299), b"leading dimension")
    refused(SHAPE, quantize(mask=P, ldmask=299), b"mask")
    refused(SHAPE, quantize(ldq=288))
    refused(SHAPE, quantize(lds=2))
    refused(SHAPE, quantize(rows=(1 << 24) + 1))
    refused(SHAPE, quantize(rows=1 << 24, cols=1 << 24, ldx=1 << 24, ldq=1 << 24, lds=1 << 17), b"2")
    refused(SHAPE, quantize(ldq=(1 << 22) + 16), b"leading dimension")
    refused(ALLOC, quantize(x=P + 2), b"element")
    refused(ALLOC, quantize(q=P + 8), b"16-byte")
    refused(ALLOC, quantize(ldq=392), b"16-byte")
    refused(ALLOC, quantize(scales=P + 1), b"4-byte")
    refused(ALLOC, quantize(lds=5), b"4-byte")
    refused(ALLOC, quantize(rows=200, sums=P, work=P, size=2 * 4 * 300 - 1), b"2400")
    refused(ALLOC, quantize(rows=200, sums=P, work=P + 64, size=1 << 20), b"256-byte")
    assert quantize(rows=0) == 0 and quantize(cols=0, ldx=0) == 0
    assert api.lib().slp_quantize_workspace_bytes(129, 5) == 40 and api.lib().slp_quantize_workspace_bytes(-1, 5) == 0


def product(**kw):
    a = dict(a=P, lda=304, sa=P, ldsa=4, ba=1, b=P, ldb=304, sb=P, ldsb=4, bb=128, bias=None, relu=0, m=5, n=7, k=300, out=P, ldo=7, dt=0, work=P, size=1 << 40)
    a.update(kw)
    return api.lib().slp_product(*a.values(), None)


def test_product():
    refused(ARG, product(a=None), b"values")
    refused(ARG, product(sb=None), b"scales")
    refused(ARG, product(out=None), b"null")
    refused(ARG, product(dt=-1), b"dtype")
    refused(ARG, product(ba=0), b"blocks")
    refused(ARG, product(bb=2), b"blocks")
    refused(ARG, product(k=-1), b"negative")
    refused(SHAPE, product(ldo=6), b"out")
    refused(SHAPE, product(lda=288), b"of a")
    refused(SHAPE, product(ldsb=0), b"of b")
    refused(SHAPE, product(m=1 << 24, n=1 << 24, ldo=1 << 24), b"matrix")
    refused(ALLOC, product(b=P + 4), b"16-byte")
    refused(ALLOC, product(ldb=312), b"16-byte")
    refused(ALLOC, product(ldsa=6), b"4-byte")
    refused(ALLOC, product(out=P + 1), b"element")
    refused(ALLOC, product(bias=P + 2), b"bias")
    need = api.lib().slp_product_workspace_bytes(100, 64, 16384)
    assert need > 0
    big = dict(m=100, n=64, k=16384, lda=16384, ldb=16384, ldsa=128, ldsb=128, ldo=64)
    refused(ALLOC, product(**big, size=need - 1), b"workspace")
    refused(ALLOC, product(**big, work=None), b"workspace")
    assert product(m=0) == 0 and product(n=0, ldo=0) == 0
    assert api.lib().slp_product_workspace_bytes(-4, 64, 64) == 0


def norm(**kw):
    a = dict(x=P, ldx=300, r=None, ldr=0, gamma=None, eps=1e-6, dt=1, rows=4, dim=300, h=None, ldh=0, y=None, ldy=0, q=P, ldq=304, scales=P, lds=4, rstd=None)
    a.update(kw)
    return api.lib().slp_rmsnorm(*a.values(), None)


def test_rmsnorm():
    refused(ARG, norm(x=None), b"null")
    refused(ARG, norm(dt=7), b"dtype")
    refused(ARG, norm(eps=-1.0), b"eps")
    refused(ARG, norm(eps=float("nan")), b"eps")
    refused(ARG, norm(dim=0), b"mean")
    refused(ARG, norm(r=P, ldr=300), b"needs h")
    refused(ARG, norm(scales=None), b"scales")
    refused(SHAPE, norm(ldx=200), b"of x")
    refused(SHAPE, norm(y=P, ldy=200), b"of y")
    refused(SHAPE, norm(r=P, ldr=300, h=P, ldh=1), b"of h")
    refused(ALLOC, norm(x=P + 1), b"element")
    refused(ALLOC, norm(gamma=P + 2), b"gamma")
    refused(ALLOC, norm(q=P + 1), b"16-byte")
    assert norm(rows=0) == 0


def norm_back(**kw):
    a = dict(dy=P, lddy=300, h=P, ldh=300, gamma=P, rstd=P, dh=None, lddh=0, dt=1, rows=200, dim=300, dx=P, lddx=300, dgamma=P, work=P, size=1 << 40)
    a.update(kw)
    return api.lib().slp_rmsnorm_backward(*a.values(), None)


def test_rmsnorm_backward():
    for name in ("dy", "h", "rstd", "dx"):
        refused(ARG, norm_back(**{name: None}), b"null")
    refused(ARG, norm_back(dt=3), b"dtype")
    refused(ARG, norm_back(dim=0), b"mean")
    refused(SHAPE, norm_back(lddx=299), b"dx")
    refused(SHAPE, norm_back(dh=P, lddh=2), b"dh")
    refused(ALLOC, norm_back(size=16), b"workspace")
    refused(ALLOC, norm_back(work=P + 128), b"workspace")
    refused(ALLOC, norm_back(dgamma=P + 1), b"element")
    assert norm_back(rows=0, dgamma=None) == 0


def test_clip():
    L = api.lib()

    def call(ptrs=(P, P), out=None, counts=(5, 6), dts=(0, 1), n=2, max_norm=1.0, norm=P, work=P, size=1 << 20):
        arr = lambda t, v: (t * len(v))(*v) if v is not None else None  # noqa: E731
        a = arr(ctypes.c_void_p, ptrs), arr(ctypes.c_int64, counts), arr(ctypes.c_int, dts)
        return (L.slp_clip_gradients(a[0], arr(ctypes.c_void_p, out), a[1], a[2], n, max_norm, norm, work, size, None),
                lambda: L.slp_gradient_norm(a[0], a[1], a[2], n, norm, work, size, None))

    refused(ARG, call(max_norm=0.0)[0], b"max_norm")
    refused(ARG, call(max_norm=float("nan"))[0], b"max_norm")
    refused(ARG, call(norm=None)[1](), b"null")
    for get in (lambda **kw: call(**kw)[0], lambda **kw: call(**kw)[1]()):
        refused(ARG, get(n=-1), b"negative")
        refused(ARG, get(ptrs=None), b"null")
        refused(ARG, get(ptrs=(P, None)), b"tensor 1")
        refused(ARG, get(counts=(5, -6)), b"negative")
        refused(ARG, get(dts=(0, 4)), b"dtype")
        refused(SHAPE, get(counts=(1 << 44, 6)), b"elements")
        refused(ALLOC, get(ptrs=(P + 2, P)), b"tensor 0")
        refused(ALLOC, get(size=8 - 1), b"workspace")
        refused(ALLOC, get(work=None), b"workspace")
    refused(ARG, call(out=(P, None))[0], b"tensor 1")
    refused(ALLOC, call(out=(P, P + 1))[0], b"tensor 1")


@pytest.mark.parametrize("rows,cols,block", [(3, 300, 1), (300, 4096, 128), (1, 1, 1), (0, 5, 1)])
def test_room_for_a_matrix_meets_the_rules(rows, cols, block):
    q, scales, b = api.empty_quantized(rows, cols, block, device="cpu")
    assert q.shape == (rows, cols) and q.stride(0) % 16 == 0 and (q.stride(0) * q.element_size()) % 4096 != 0 and b == block
    assert scales.shape == (-(-rows // block), -(-cols // 128)) and scales.stride(0) % 4 == 0
