"""The operators' binding: whose memory and streams a call uses, which matrices it takes."""

import numpy as np
import pytest
import torch

from paper_2403_11204_amd import api

pytestmark = pytest.mark.gpu
DEV = "cuda"


def test_tensors_that_only_the_call_holds():
    """An iterator's tensors live until the call has been queued: nothing that the call allocates lies in their memory."""
    halves = [torch.full((n,), 0.5, dtype=torch.bfloat16, device=DEV) for n in (64, 128, 256, 64, 512)]
    ref = np.sqrt(sum(0.25 * h.numel() for h in halves))
    for _ in range(5):
        assert abs(float(api.gradient_norm(h.float() for h in halves)) - ref) <= 1e-6 * ref
        assert abs(float(api.gradient_norm(map(torch.clone, halves))) - ref) <= 1e-6 * ref
        out = [torch.empty(h.shape, device=DEV) for h in halves]
        norm = api.clip_gradients((h.float() for h in halves), ref / 2, out=iter(out))
        assert abs(float(norm) - ref) <= 1e-6 * ref and all(bool(((o - 0.25).abs() <= 1e-6).all()) for o in out)
