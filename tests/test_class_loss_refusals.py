"""What the losses over a linear layer's classes refuse, before any device is touched.  CPU only."""

import pytest

from paper_2403_11204_amd import api

P = 0x100000          # an address that is never followed
ARG, SHAPE, ALLOC = -1, -2, -3


def refused(code, got, word=None):
    assert got == code, (got, api.lib().slp_last_error())
    if word:
        assert word in api.lib().slp_last_error(), api.lib().slp_last_error()


OUT = dict(scale=1.0, loss=P, losses=P, lse=P, dx=P, lddx=64, dw=P, lddw=64, dw_dt=0, dbias=P, work=P, size=1 << 60)


def xent(**kw):
    a = dict(x=P, ldx=64, w=P, ldw=64, bias=P, dt=0, rows=10, classes=300, dim=64, y=P, id_bytes=4, **OUT)
    a.update(kw)
    return api.lib().slp_linear_cross_entropy(*a.values(), None)


def distil(**kw):
    a = dict(x=P, ldx=64, w=P, ldw=64, bias=P, dt=0, rows=10, classes=300, dim=64, top=P, ldtop=8, top_dt=0, ids=P, ldids=8, id_bytes=4, k=8, t=2.0, **OUT)
    a.update(kw)
    return api.lib().slp_linear_distillation(*a.values(), None)


@pytest.mark.parametrize("call", [xent, distil])
def test_common(call):
    for name in ("x", "w", "loss", "losses", "lse"):
        refused(ARG, call(**{name: None}), b"null")
    refused(ARG, call(dt=2), b"dtype")
    refused(ARG, call(dw_dt=-1), b"dtype")
    refused(ARG, call(rows=-1), b"rows")
    refused(ARG, call(classes=0), b"classes")
    refused(ARG, call(dim=0), b"dim")
    refused(ARG, call(id_bytes=2), b"4 or 8")
    refused(ARG, call(scale=float("nan")), b"finite")
    refused(ARG, call(scale=float("inf")), b"finite")
    refused(SHAPE, call(ldx=63), b"of x")
    refused(SHAPE, call(ldw=63), b"of w")
    refused(SHAPE, call(lddx=63), b"dx")
    refused(SHAPE, call(lddw=63), b"dw")
    refused(SHAPE, call(ldx=(1 << 20) + 4), b"apart")
    refused(SHAPE, call(ldw=(1 << 20) + 4), b"apart")
    refused(SHAPE, call(rows=(1 << 20) + 1))
    refused(SHAPE, call(classes=(1 << 24) + 1))
    refused(SHAPE, call(dim=1 << 20, classes=1 << 14, ldx=1 << 20, ldw=1 << 20, lddx=1 << 20, lddw=1 << 20))
    refused(SHAPE, call(rows=1 << 20, classes=1 << 20))
    refused(ALLOC, call(x=P + 2), b"x")
    refused(ALLOC, call(dx=P + 2), b"dx")
    refused(ALLOC, call(bias=P + 2), b"vector")
    refused(ALLOC, call(lse=P + 1), b"vector")
    refused(ALLOC, call(dt=1, w=P + 1), b"w")
    refused(ALLOC, call(work=None), b"workspace")
    refused(ALLOC, call(work=P + 128), b"256-byte")
    need = api.lib().slp_linear_loss_workspace_bytes(P, 64, P, 64, 0, 10, 300, 64, 8 if call is distil else 0, 7)
    assert need > 0
    refused(ALLOC, call(size=need - 1), b"workspace")


def test_targets():
    refused(ARG, xent(y=None), b"null")
    refused(ALLOC, xent(y=P + 4, id_bytes=8), b"ids")
    refused(ARG, distil(ids=None), b"null")
    refused(ARG, distil(top=None), b"null")
    refused(ARG, distil(top_dt=7), b"dtype")
    refused(ARG, distil(k=0), b"teacher")
    refused(ARG, distil(k=1025, ldtop=1025, ldids=1025), b"teacher")
    refused(ARG, distil(t=0.0), b"temperature")
    refused(ARG, distil(t=float("nan")), b"temperature")
    refused(ARG, distil(t=-1.0), b"temperature")
    refused(SHAPE, distil(ldtop=7), b"top")
    refused(SHAPE, distil(ldids=7), b"classes")
    refused(ALLOC, distil(top=P + 2), b"top")
    refused(SHAPE, distil(rows=1 << 16, k=1024, ldtop=1024, ldids=1024), b"targets")


def test_workspace():
    size = api.lib().slp_linear_loss_workspace_bytes
    a = (P, 4096, P, 4096, 1, 8192, 131072, 4096, 0)
    assert size(*a, 0) < size(*a, 1) < size(*a, 3) < size(*a, 7)
    assert size(*a, 7) < 8192 * 131072 * 2                       # less than the logits alone in 16 bits
    b = (P, 4096, P, 4096, 1, 65536, 131072, 4096, 0)
    assert size(*b, 7) < size(*a, 7) + 65536 * 4096 * (4 + 2) + (2 << 30)     # what grows with the rows: x's gradient, its copy, statistics
    assert size(P + 2, *a[1:], 0) > size(*a, 0)                  # a copy of what cannot be read in place
    assert size(P, 64, P, 64, 9, 10, 300, 64, 0, 7) == 0 and size(P, 64, P, 64, 0, 0, 300, 64, 0, 7) == 0 and size(P, 64, P, 64, 0, 10, 300, 64, 1025, 7) == 0
