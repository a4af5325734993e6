"""The operators' example in README.md runs as it stands and gives the gradients of what it computes."""

import os
import re

import pytest
import torch

from paper_2403_11204_amd import api

pytestmark = pytest.mark.gpu
DEV = "cuda"


def test_the_example():
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")).read()
    block = re.search(r"\n\n((?:    .*\n)*    w = api\.quantize(?:.*\n)(?:    .*\n)*)", text).group(1)
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    M, N, K = 70, 200, 300
    randn = lambda *s: torch.randn(*s, device=DEV, generator=g)  # noqa: E731
    have = {"api": api, "W": randn(N, K) / K ** 0.5, "b": randn(N), "gamma": 1 + 0.1 * randn(K), "x": randn(M, K).bfloat16(), "h": randn(M, K).bfloat16(), "dz": randn(M, N).bfloat16(),
            "d": randn(M, K).bfloat16()}
    norms = {k: v.clone() for k, v in have.items() if torch.is_tensor(v)}
    have["max_norm"] = 1e9
    exec(re.sub(r"^    ", "", block, flags=re.M).replace("max_norm=1.0", "max_norm=max_norm"), have)
    # beside differentiation without any rounding: 8 bits are 2.6 % off in the mean square
    t = {k: v.double().requires_grad_() for k, v in norms.items()}
    s = t["x"] + t["h"]
    y = s / torch.sqrt((s * s).mean(1, keepdim=True) + 1e-6) * t["gamma"]
    z = torch.relu(torch.addmm(t["b"], y, t["W"].t().contiguous()))
    (z * t["dz"].detach()).sum().add((s * t["d"].detach()).sum()).backward()
    for got, ref in ((have["dW"], t["W"].grad), (have["g"].column_sums, t["b"].grad), (have["dgamma"], t["gamma"].grad), (have["dx"], t["x"].grad)):
        assert float(torch.nn.functional.cosine_similarity(got.double().flatten(), ref.flatten(), dim=0)) > 0.97
    assert float(have["norm"]) > 0
