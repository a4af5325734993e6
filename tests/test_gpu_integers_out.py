"""Rows quantised into integers that are there already."""

import pytest
import torch

from paper_2403_11204_amd import api

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 40), (3, 7), (30, 301), (200, 4096), (2, 20000), (0, 9)])
def test_into_the_same(rows, cols, dtype):
    g = torch.Generator().manual_seed(rows + cols)
    x, other = (torch.randn(rows, cols, generator=g).to(dtype).cuda() for _ in range(2))
    want, out = api.quantize_integers(x), api.quantize_integers(other)
    r = api.quantize_integers(x, out=out)
    assert r.q is out.q and r.scales is out.scales and torch.equal(out.q, want.q) and torch.equal(out.scales, want.scales)


def test_into_a_wider_matrix():
    x = torch.randn(20, 40, device="cuda")
    want = api.quantize_integers(x)
    wide, scales = torch.full((41, 96), 77, dtype=torch.int8, device="cuda"), torch.full((22,), 5.0, device="cuda")
    api.quantize_integers(x, out=api.Integers(wide[1:41:2, 16:56], scales[1:21]))
    assert torch.equal(wide[1:41:2, 16:56], want.q) and torch.equal(scales[1:21], want.scales) and scales[0] == 5 and scales[21] == 5
    assert not wide[1:41:2, 56:64].any()                                  # zeros up to the next multiple of 16
    assert (wide[::2] == 77).all() and (wide[:, :16] == 77).all() and (wide[:, 64:] == 77).all()


def test_refused():
    x = torch.randn(4, 40, device="cuda")
    q, s = (lambda *size: torch.zeros(*size, dtype=torch.int8, device="cuda")), torch.zeros(4, device="cuda")
    one = q(1, 40)                                                         # (40 bytes: the row's 48 do not fit)
    for bad in (lambda: api.quantize_integers(x, out=(q(5, 48)[:, :40], torch.zeros(5, device="cuda"))), lambda: api.quantize_integers(x, out=(q(4, 41), s)), lambda: api.quantize_integers(x, out=(q(4, 48)[:, :40], s[:3])),
                lambda: api.quantize_integers(x, out=(q(4, 48)[:, :40].float(), s)), lambda: api.quantize_integers(x, out=(q(4, 48)[:, :40], None)), lambda: api.quantize_integers(x, out=(q(4, 48)[:, :40].cpu(), s)),
                lambda: api.quantize_integers(x, out=(q(4, 48)[:, :40], s.double())), lambda: api.quantize_integers(x, out=(q(40, 4).t(), s)), lambda: api.quantize_integers(x[:1], out=(one, s[:1])),
                lambda: api.quantize_integers(x, out=(q(8, 80)[4:, 40:], s))):
        with pytest.raises(AssertionError):
            bad()
    for bad in (lambda: api.quantize_integers(x, out=(q(4, 40), s)), lambda: api.quantize_integers(x, out=(q(4, 56)[:, 8:48], s)), lambda: api.quantize_integers(x, out=(q(5, 64)[:4, 8:48], s))):
        with pytest.raises((api.SlpError, AssertionError)):
            bad()
