"""Losses whose logits beyond 1 GiB are computed again for the gradient: kept and recomputed pieces together against 64 bits on the device, classes and biases in all of them.

The recomputed pieces of bf16 rows of more than two k-tiles run on 256x256 tiles, the others on 128x128; few rows on 64x64 (bf16) and 32x64 (float32)."""

import pytest
import torch

import test_gpu_class_loss_large as large

pytestmark = pytest.mark.gpu


# 3 pieces, 2 of them kept; the same with copies of x and W; a distillation; a last row and class alone in their tiles; 5, 2; one k-tile; float32 5, 4, and with copies; few rows 16, 12; 3, 2
@pytest.mark.parametrize("rows,classes,dim,k,bias,dtype", [(5003, 60001, 264, 0, True, "bf16"), (5003, 60001, 261, 0, True, "bf16"), (8200, 40008, 200, 3, True, "bf16"), (4865, 60417, 192, 2, True, "bf16"),
                                                           (16385, 33001, 136, 0, False, "bf16"), (5003, 60001, 40, 0, True, "bf16"), (4100, 66001, 132, 0, True, "fp32"), (4100, 66001, 71, 2, True, "fp32"),
                                                           (20, 16777213, 16, 0, True, "bf16"), (20, 16777213, 8, 2, True, "fp32"), (100, 3000001, 72, 0, True, "bf16")])
def test_recomputed(rows, classes, dim, k, bias, dtype):
    large.test_large(rows, classes, dim, k, bias, dtype)
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype,dim", [("bf16", 264), ("fp32", 68)])
def test_labels_of_one_piece(dtype, dim):
    """All of the rows' own classes in the last piece, or all in the first: what is taken from P at a class is taken there and nowhere else."""
    from paper_2403_11204_amd import api
    rows, classes = 5003, 60001
    g = torch.Generator(device="cuda").manual_seed(7)
    x = torch.randn(rows, dim, device="cuda", generator=g).to(large.DT[dtype])
    w = (torch.randn(classes, dim, device="cuda", generator=g) * (2.5 / dim ** 0.5)).to(large.DT[dtype])
    W, z = w.double(), x.double() @ w.double().t()
    soft = torch.softmax(z, 1)
    # logits: 6 standard deviations of dim roundings of |z| + 7.5 by 2^-24; P's error twice that and 2^-22 of it, half a step of bf16 behind; dw's 5003 additions and half step
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    dz = 6 * dim ** 0.5 * 2.0 ** -24 * (float(z.abs().max()) + 7.5)
    for first, last in ((classes - 300, classes), (0, 300), (classes - 1, classes)):
        y = torch.randint(first, last, (rows,), device="cuda", generator=g)
        r = api.linear_cross_entropy(x, w, y, dtype=api.F32)
        G = soft.scatter_add(1, y[:, None], torch.full((rows, 1), -1.0, dtype=torch.float64, device="cuda")) / rows
        err = (2 * dz + 2.0 ** -22) * soft / rows + (half if dtype == "bf16" else 2.0 ** -23) * G.abs()
        err.scatter_add_(1, y[:, None], torch.full((rows, 1), 2.0 ** -22 / rows, dtype=torch.float64, device="cuda"))
        Gt, X = G.t().contiguous(), x.double()
        off = (r.dw.double() - Gt @ X).abs() - (err.t().contiguous() @ X.abs() + 6 * rows ** 0.5 * 2.0 ** -24 * (Gt.abs() @ X.abs()) + 2.0 ** -23 * (Gt @ X).abs() + 1e-30)
        assert off.max() <= 0, (first, float(off.max()))
        off = (r.dx.double() - G @ W).abs() - (err @ W.abs() + 6 * classes ** 0.5 * 2.0 ** -24 * (G.abs() @ W.abs()) + 1.01 * half * (G @ W).abs() + 1e-30)
        assert off.max() <= 0, (first, float(off.max()))
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype,dim,k", [("bf16", 264, 0), ("bf16", 264, 2), ("bf16", 40, 0), ("fp32", 68, 0), ("bf16", 261, 0)])
def test_padding_and_masked_classes(dtype, dim, k):
    """Rows that do not count hold anything, classes that the bias leaves out have no gradient, a row with a NaN reaches its own, in all pieces; and the same bits every time."""
    from paper_2403_11204_amd import api
    rows, classes, masked = 5003, 60001, torch.tensor([0, 5, 20223, 20224, 45000, 59999, 60000], device="cuda")
    g = torch.Generator(device="cuda").manual_seed(9)
    x = torch.randn(rows, dim, device="cuda", generator=g).to(large.DT[dtype])
    w = (torch.randn(classes, dim, device="cuda", generator=g) * (2.5 / dim ** 0.5)).to(large.DT[dtype])
    b = torch.randn(classes, device="cuda", generator=g)
    b[masked] = -float("inf")
    ids = torch.randint(6, 20000, (rows, max(k, 1)), device="cuda", generator=g)
    ids[2500:] += 25000                                                    # (the second and the third piece; none of the masked)
    ids[ids == 45000] += 1
    padding = torch.arange(0, rows, 17, device="cuda")
    ids[padding] = -1
    top = torch.randn(rows, k, device="cuda", generator=g) if k else None
    call = lambda x: api.linear_distillation(x, w, top, ids, bias=b, temperature=2.0) if k else api.linear_cross_entropy(x, w, ids[:, 0].contiguous(), bias=b)  # noqa: E731
    r = call(x)
    assert all(torch.isfinite(t).all() for t in r)
    assert not r.dw[masked].any() and not r.dbias[masked].any() and not r.dx[padding].any() and not r.losses[padding].any()
    for value in (float("nan"), float("inf")):
        y = x.clone()
        y[padding] = value
        again = call(y)
        for name in ("loss", "losses", "dx", "dw", "dbias"):
            assert torch.equal(getattr(r, name), getattr(again, name)), name
    assert all(torch.equal(u, v) for u, v in zip(r, call(x)))
    x[1, 3] = float("nan")                                                 # a row that counts
    bad = call(x)
    others = torch.arange(rows, device="cuda") != 1
    assert bad.loss.isnan() and bad.dx[1].isnan().all() and bad.dw.isnan().all() and bad.dbias.isnan().all()
    assert torch.equal(bad.dx[others], r.dx[others]) and torch.equal(bad.losses[others], r.losses[others])
    torch.cuda.empty_cache()
