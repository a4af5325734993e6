"""What pipeline.py does with the residual segment as a left partition besides training it."""

import pytest
import torch

from paper_2403_11204_amd import api, pipeline
from paper_2403_11204_amd.residual import ResidualSegment

pytestmark = pytest.mark.gpu
DEV = "cuda"


def test_stored_and_joined():
    left = ResidualSegment(128, 200, 2, seed=5)
    right = api.Segment([128, 64, 10], api.RELU_HIDDEN_IDENTITY_LAST, api.SOFTMAX_XENT, max_batch=50, dtype=api.BF16)
    right.init(3)
    X = torch.randn(130, 128, device=DEV).bfloat16()
    parts = [X[a:a + 50] for a in range(0, 130, 50)]
    stored = pipeline.store_response(left, X, batch=50)
    assert torch.equal(stored, torch.cat([left.forward(p) for p in parts]))
    joined = pipeline.joined_forward([left, right], X, batch=50)
    assert torch.equal(joined, torch.cat([right.forward(left.forward(p)) for p in parts]))
