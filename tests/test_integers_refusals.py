"""Integers: what is refused before any device is touched, and the oracle's own pins.  CPU only."""

import numpy as np

from oracle import integers
from paper_2403_11204_amd import api

P = 0x100000          # an address that is never followed
ARG, SHAPE, ALLOC = -1, -2, -3


def refused(code, got, word=None):
    assert got == code, (got, api.lib().slp_last_error())
    if word:
        assert word in api.lib().slp_last_error(), api.lib().slp_last_error()


def quantize(**kw):
    a = dict(x=P, ldx=300, dt=0, rows=10, cols=300, q=P, ldq=304, scales=P)
    a.update(kw)
    return api.lib().slp_quantize_integers(*a.values(), None)


def product(**kw):
    a = dict(a=P, lda=304, sa=P, b=P, ldb=304, sb=P, bias=None, relu=0, m=5, n=7, k=300, out=P, ldo=7, dt=0, work=P, size=1 << 40)
    a.update(kw)
    return api.lib().slp_product_integers(*a.values(), None)


def test_quantize():
    refused(ARG, quantize(x=None), b"null")
    refused(ARG, quantize(q=None), b"null")
    refused(ARG, quantize(scales=None), b"null")
    refused(ARG, quantize(dt=3), b"dtype")
    refused(ARG, quantize(rows=-1), b"negative")
    refused(SHAPE, quantize(ldx=299), b"of x")
    refused(SHAPE, quantize(ldq=288), b"of q")
    refused(SHAPE, quantize(rows=1 << 24, cols=1 << 24, ldx=1 << 24, ldq=1 << 24))
    refused(ALLOC, quantize(q=P + 8), b"16-byte")
    refused(ALLOC, quantize(ldq=312), b"16-byte")
    refused(ALLOC, quantize(x=P + 1), b"x")
    refused(ALLOC, quantize(scales=P + 2), b"scales")
    assert quantize(rows=0) == 0


def test_product():
    for name in ("a", "b", "sa", "sb", "out"):
        refused(ARG, product(**{name: None}), b"null")
    refused(ARG, product(dt=16), b"dtype")
    refused(ARG, product(k=-1), b"negative")
    refused(SHAPE, product(k=131072, lda=131072, ldb=131072), b"131071")
    refused(SHAPE, product(ldo=6), b"out")
    refused(SHAPE, product(lda=288), b"of a")
    refused(SHAPE, product(m=1 << 24, n=1 << 24, ldo=1 << 24), b"matrix")
    refused(ALLOC, product(b=P + 4), b"16-byte")
    refused(ALLOC, product(ldb=312), b"16-byte")
    refused(ALLOC, product(out=P + 1), b"element")
    refused(ALLOC, product(bias=P + 2), b"bias")
    need = api.lib().slp_product_integers_workspace_bytes(100, 64, 16384)
    assert need > 0 and api.lib().slp_product_integers_workspace_bytes(100, 64, 131072) == 0
    big = dict(m=100, n=64, k=16384, lda=16384, ldb=16384, ldo=64)
    refused(ALLOC, product(**big, size=need - 1), b"workspace")
    refused(ALLOC, product(**big, work=P + 64), b"256-byte")
    assert product(m=0) == 0 and product(n=0, ldo=0) == 0


def test_oracle():
    q, s = integers.quantize(np.array([[127.0, 0.5, 1.5, 2.5, -0.5, -126.5], [0, 0, 0, 0, 0, 0], [2.0, -2.0, 1.0, 0.0, 0.0, np.nan]]))
    assert q[0].tolist() == [127, 0, 2, 2, 0, -126] and s[0] == 1 and s[1] == 0 and not q[1:].any() and np.isnan(s[2])
    out = integers.product(np.array([[1, -2]]), [0.5], np.array([[3, 4], [-1, 1]]), [2.0, 1.0], [0.0, 1.0], relu=True)
    assert out.tolist() == [[0.0, 0.0]]
    assert integers.product(np.array([[1, -2]]), [0.5], np.array([[3, 4], [-1, 1]]), [2.0, 1.0]).tolist() == [[-5.0, -1.5]]
