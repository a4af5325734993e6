"""More of what the 8-bit operators refuse before any device is touched.  CPU only."""

from paper_2403_11204_amd import api
from test_eightbit_arguments import ALLOC, ARG, P, product, quantize, refused


def test_sums_of_no_rows_on_no_boundary():
    refused(ALLOC, quantize(rows=0, sums=P + 2), b"element")


def test_float32_sums_go_with_the_two_types_only():
    assert product(dt=api.BF16 | 16, m=0) == 0 and product(dt=api.F32 | 16, m=0) == 0
    refused(ARG, product(dt=2 | 16), b"dtype")
    refused(ARG, product(dt=-16), b"dtype")
    refused(ALLOC, product(dt=api.BF16 | 16, out=P + 1), b"element")
