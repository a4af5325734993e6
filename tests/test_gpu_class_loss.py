"""Losses over a linear layer's classes against the oracle in 64 bits.

Tolerances, per element.  A logit of the operands adds dim exact products in float32: each addition rounds by 2^-24 of a partial sum, which stays below
`most` = |z| + 3 sqrt(sum of the squared products); dim such roundings of random sign come to sqrt(dim) 2^-24 most, of which 6 are allowed (float32
operands: three parts of 8 bits, what is left out is below 3 * 2^-26 of each product, inside the same).  With that error dz of the logits:
    lse, losses    2 dz + 2^-21 (their size and the logits'), exponential and logarithm 2 steps each;  loss: their mean's, 2^-23 more
    P              p (2 dz + 2^-22) and, in bf16, half a step 2^-8 of the value behind the target's subtraction; at a target besides its own probability's
                   error 2^-24 (|log p| + k / 2 + 4) of it: the difference to the largest entry, its exponential, the sum of k, the quotient
    dx             |P's error| |W| + sqrt(terms) 2^-24 times 6 of the sum of sizes, and the output's half step;  dw the same with |x|
    dbias          |p's error| summed, 2^-24 of each part's sum, 2^-40 of each row
"""

import numpy as np
import pytest
import torch

from oracle import class_loss
from paper_2403_11204_amd import api

pytestmark = pytest.mark.gpu
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}
HALF = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8}


def _f64(t):
    return t.detach().cpu().double().numpy()


def check(r, x, w, ids, top=None, bias=None, temperature=1.0, scale=1.0, dtype="fp32", dw_dtype=None, gradients=True, weights=True, rows=None):
    """r against the oracle; rows: those that are compared (None: all)."""
    dw_dtype = dw_dtype or dtype
    X, W, B = _f64(x), _f64(w), None if bias is None else _f64(bias)
    C = ids.cpu().numpy().reshape(x.shape[0], -1)
    o = class_loss.loss(np.where(np.isfinite(X), X, 0.0), W, C, None if top is None else _f64(top), B, temperature, scale)
    dim, n = X.shape[1], max(1, int(o["counts"].sum()))
    z = np.log(np.maximum(o["p"], 1e-300)) + o["lse"][:, None]
    most = (np.abs(np.where(o["p"] > 0, z, 0.0)) * temperature + 3 * np.sqrt((X * X) @ (W * W).T)).max(1)
    most = np.where(np.isfinite(most), most, 0.0)
    dz = 6 * np.sqrt(dim) * 2.0 ** -24 * most / temperature + 2.0 ** -23 * (np.abs(o["lse"]) + most)
    c = o["counts"]
    live = np.isfinite(X).all(1)
    size = np.abs(o["lse"]) + np.abs(o["losses"]) / temperature ** 2 + most
    tol = temperature ** 2 * (2 * dz + 2.0 ** -21 * size)
    assert (np.abs(_f64(r.lse) - o["lse"]) <= tol / temperature ** 2)[live].all()
    assert (np.abs(_f64(r.losses) - o["losses"]) <= np.where(c, tol, 0.0)).all()
    assert abs(float(r.loss) - o["loss"]) <= (tol[c].mean() if c.any() else 0.0) + 2.0 ** -23 * abs(o["loss"])
    if not gradients:
        assert r.dx is None and r.dw is None and r.dbias is None
        return
    a = abs(scale) * temperature / n
    X = np.where(c[:, None], X, 0.0)
    g = np.abs(o["dz"])
    target = np.abs(o["p"] * a - o["dz"] * np.sign(scale))             # the targets' probabilities times a
    t_err = 2.0 ** -24 * target * (np.abs(np.log(np.maximum(target / a, 1e-30))) + C.shape[1] / 2 + 4)
    p_err = np.where(c[:, None], a * o["p"] * (2 * dz[:, None] + 2.0 ** -22) + 2.0 ** -23 * g + t_err, 0.0)
    P_err = p_err + (2.0 ** -8 * g if dtype == "bf16" else 0.0)

    def product(err, left, right, got, want, half):
        terms = left.shape[1]
        tol = err @ np.abs(right) + 6 * np.sqrt(terms) * 2.0 ** -24 * (np.abs(left) @ np.abs(right)) + half * np.abs(want) + 1e-37
        far = np.abs(_f64(got) - want) - tol
        assert (far <= 0).all(), (float(far.max()), np.unravel_index(far.argmax(), far.shape))

    product(P_err, g, W, r.dx, o["dx"], 1.01 * HALF[dtype])
    assert (_f64(r.dx)[~c] == 0).all() and r.dx.dtype == x.dtype
    if not weights:
        assert r.dw is None and r.dbias is None
        return
    assert r.dw.dtype == DT[dw_dtype]
    product(P_err.T, g.T, X, r.dw, o["dw"], 1.01 * HALF[dw_dtype])
    if bias is None:
        assert r.dbias is None
    else:
        tol = p_err.sum(0) + 2.0 ** -22 * g.sum(0) + 2.0 ** -23 * a * o["p"][c].sum(0) + a * 2.0 ** -40 * n + 2.0 ** -23 * np.abs(o["dbias"])
        assert (np.abs(_f64(r.dbias) - o["dbias"]) <= tol).all()


def make(seed, rows, classes, dim, dtype, bias=True, k=0, missing=0.2, long_ids=False):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, dim, generator=g).to(DT[dtype]).cuda()
    w = (torch.randn(classes, dim, generator=g) * (2.5 / dim ** 0.5)).to(DT[dtype]).cuda()
    b = torch.randn(classes, generator=g).cuda() if bias else None
    ids = torch.randint(classes, (rows, max(k, 1)), generator=g, dtype=torch.int64 if long_ids else torch.int32)
    ids = torch.where(torch.rand(rows, max(k, 1), generator=g) < missing, torch.full_like(ids, -1), ids)
    if k == 0:
        return x, w, b, ids[:, 0].contiguous().cuda(), None
    return x, w, b, ids.cuda(), (3 * torch.randn(rows, k, generator=g)).to(DT[dtype]).cuda()


SIZES = [(1, 1, 1), (1, 2, 3), (3, 7, 5), (16, 64, 64), (17, 65, 100), (64, 129, 8), (65, 1000, 333), (130, 257, 1), (300, 47, 60), (257, 2049, 136), (1, 5001, 512), (700, 16, 24),
         (1410, 47, 60), (33, 3001, 777)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,classes,dim", SIZES)
def test_cross_entropy(rows, classes, dim, dtype):
    x, w, b, y, _ = make(rows + classes, rows, classes, dim, dtype, missing=0.2 if rows > 3 else 0.0)
    check(api.linear_cross_entropy(x, w, y, bias=b), x, w, y, bias=b, dtype=dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,classes,dim,k,temperature", [(1, 1, 1, 1, 1.0), (3, 7, 5, 7, 2.0), (17, 65, 100, 1, 1.0), (64, 129, 8, 8, 4.0), (65, 1000, 333, 33, 0.5), (130, 47, 60, 16, 3.0),
                                                            (300, 2049, 136, 100, 1.0), (5, 300, 24, 1024, 2.0)])
def test_distillation(rows, classes, dim, k, temperature, dtype):
    x, w, b, ids, top = make(rows + classes, rows, classes, dim, dtype, k=k, missing=0.2 if rows > 1 else 0.0, long_ids=rows % 2 == 1)
    check(api.linear_distillation(x, w, top, ids, bias=b, temperature=temperature), x, w, ids, top, b, temperature, dtype=dtype)


@pytest.mark.parametrize("gradients,weights", [(False, True), (True, False)])
def test_what_is_asked_for(gradients, weights):
    x, w, b, y, _ = make(1, 70, 300, 64, "bf16")
    check(api.linear_cross_entropy(x, w, y, bias=b, gradients=gradients, weight_gradients=weights), x, w, y, bias=b, dtype="bf16", gradients=gradients, weights=weights)
    check(api.linear_cross_entropy(x, w, y), x, w, y, dtype="bf16")
    check(api.linear_cross_entropy(x, w, y, scale=-3.0, dtype=api.F32), x, w, y, scale=-3.0, dtype="bf16", dw_dtype="fp32")
    xf, wf = x.float(), w.float()
    check(api.linear_cross_entropy(xf, wf, y, dtype=api.BF16), xf, wf, y, dtype="fp32", dw_dtype="bf16")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_strides_and_alignments(dtype):
    x, w, b, ids, top = make(5, 70, 300, 64, dtype, k=6, long_ids=True)
    want = api.linear_distillation(x, w, top, ids, bias=b, temperature=2.0)
    for pad, first in ((8, 0), (1, 0), (8, 1), (8, 4), (0, 0)):
        wide = lambda t, f: torch.full((t.shape[0], t.shape[1] + pad + f), float("nan"), device="cuda").to(t.dtype)  # noqa: E731
        xs, ws = wide(x, first), wide(w, first)
        xs[:, first:first + 64], ws[:, first:first + 64] = x, w
        tops, idss = wide(top, first), torch.full((70, 6 + pad + first), 3, dtype=torch.int64, device="cuda")
        tops[:, first:first + 6], idss[:, first:first + 6] = top, ids
        got = api.linear_distillation(xs[:, first:first + 64], ws[:, first:first + 64], tops[:, first:first + 6], idss[:, first:first + 6], bias=b, temperature=2.0)
        for u, v in zip(got, want):
            assert torch.equal(u, v)
    # every other row
    got = api.linear_distillation(x.repeat_interleave(2, 0)[::2], w.repeat_interleave(2, 0)[1::2], top.repeat_interleave(2, 0)[::2], ids.repeat_interleave(2, 0)[::2], bias=b, temperature=2.0)
    for u, v in zip(got, want):
        assert torch.equal(u, v)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_and_entries_that_do_not_count(dtype):
    nan, inf = float("nan"), float("inf")
    x, w, b, y, _ = make(7, 40, 150, 72, dtype, missing=0.0)
    y[3], y[10], y[39] = -1, 150, -(1 << 31)
    x[3], x[10] = nan, inf                           # padding holds anything
    check(api.linear_cross_entropy(x, w, y, bias=b), x, w, y, bias=b, dtype=dtype)
    y64 = y.long()
    y64[10], y64[39] = 1 << 32, -(1 << 40)
    check(api.linear_cross_entropy(x, w, y64, bias=b), x, w, y64, bias=b, dtype=dtype)
    x, w, b, ids, top = make(8, 40, 150, 72, dtype, k=5, missing=0.0)
    top[0, 2], top[1] = -inf, -inf                   # an entry, all entries masked by the teacher's logits
    ids[2], top[2], x[2] = -1, nan, nan              # all by their classes
    ids[4, 1:], top[4, 1:] = -1, nan                 # a list of one
    ids[5, :] = ids[5, 0]                            # one class five times
    ids[6, 3] = ids[6, 0]
    clean = torch.where(ids >= 0, top, torch.zeros_like(top))
    check(api.linear_distillation(x, w, top, ids, bias=b, temperature=2.0), x, w, ids, clean, b, 2.0, dtype=dtype)
    none = api.linear_cross_entropy(x, w, torch.full((40,), -1, dtype=torch.int32, device="cuda"), bias=b)
    assert float(none.loss) == 0 and not none.losses.any() and not none.dx.any() and not none.dw.any() and not none.dbias.any()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_masked_classes_and_values_without_a_number(dtype):
    nan, inf = float("nan"), float("inf")
    x, w, b, y, _ = make(9, 40, 150, 72, dtype, missing=0.0)
    y.clamp_(max=99)
    b[100:] = -inf                                   # classes that the bias leaves out
    r = api.linear_cross_entropy(x, w, y, bias=b)
    part = api.linear_cross_entropy(x, w[:100], y, bias=b[:100])
    check(part, x, w[:100], y, bias=b[:100], dtype=dtype)
    assert not r.dw[100:].any() and not r.dbias[100:].any()
    assert torch.allclose(r.lse, part.lse, rtol=0, atol=2e-6) and torch.allclose(r.dbias[:100], part.dbias, rtol=1e-5, atol=1e-7)
    b[100:] = torch.finfo(torch.float32).min
    low = api.linear_cross_entropy(x, w, y, bias=b)
    for u, v in zip(low, r):
        assert torch.equal(u, v)
    b[:] = torch.finfo(torch.float32).min            # of all classes: the logits do not reach beside it, all are alike
    r = api.linear_cross_entropy(x, w, y, bias=b)
    assert torch.allclose(r.losses, torch.full_like(r.losses, np.log(150)), rtol=2e-6)
    # a target that the bias masks: infinite loss, and a gradient of -1 all the same
    b[:] = 0
    b[5] = -inf
    y[0] = 5
    r = api.linear_cross_entropy(x, w, y, bias=b)
    assert r.losses[0] == inf and r.loss == inf and torch.isfinite(r.dx).all() and torch.isfinite(r.dw).all()
    # NaN in one row: that row and what it reaches
    x[1, 3] = nan
    r = api.linear_cross_entropy(x, w, y.clamp(max=4), bias=torch.zeros_like(b))
    assert r.losses[1].isnan() and r.loss.isnan() and r.dx[1].isnan().all() and not r.dx[2:].isnan().any() and r.dw.isnan().all() and r.dbias.isnan().all()
    assert not r.losses[2:].isnan().any() and not r.lse[2:].isnan().any()


def test_logits_far_apart():
    # a class that has all the probability, and gradients that are small beside what they are differences of
    for dtype in ("bf16", "fp32"):
        x, w, b, y, _ = make(11, 64, 200, 64, dtype, missing=0.0)
        b.zero_()
        b[7] = 80.0
        y[:] = 7
        check(api.linear_cross_entropy(x, w, y, bias=b), x, w, y, bias=b, dtype=dtype)
        b[7] = 12.0
        check(api.linear_cross_entropy(x, w, y, bias=b), x, w, y, bias=b, dtype=dtype)
        y[:] = 8
        b[7] = 300.0
        check(api.linear_cross_entropy(x, w, y, bias=b), x, w, y, bias=b, dtype=dtype)


def test_no_rows():
    x, w, b, y, top = make(1, 4, 30, 24, "bf16", k=3)
    for r in (api.linear_cross_entropy(x[:0], w, y[:0, 0].contiguous(), bias=b), api.linear_distillation(x[:0], w, top[:0], y[:0], bias=b)):
        assert float(r.loss) == 0 and r.losses.numel() == 0 and r.dx.shape == (0, 24) and r.dw.shape == (30, 24) and not r.dw.any() and not r.dbias.any()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("aligned", [True, False])
def test_pieces_of_the_classes(dtype, aligned):
    """More logits than a piece holds: the pieces together are the whole, the last one shorter."""
    rows, classes, dim = (5000, 60001, 16 if aligned else 13)
    x, w, b, ids, top = make(3, rows, classes, dim, dtype, k=4)
    top[:, 1] = 2 * torch.randn(rows, generator=torch.Generator().manual_seed(1)).to(top)
    ids[:, 1] = torch.randint(59000, classes, (rows,), generator=torch.Generator().manual_seed(2)).to(ids)          # in the last piece
    r = api.linear_distillation(x, w, top, ids, bias=b, temperature=2.0)
    X, W = x.double(), w.double()
    z = (X @ W.t() + b.double()) / 2
    lse = torch.logsumexp(z, 1)
    t = torch.where(ids >= 0, top.double() / 2, torch.full_like(top, -float("inf"), dtype=torch.float64))
    p = torch.softmax(t, 1)                          # (no row is without an entry: the second one always counts)
    losses = 4 * (p * torch.where(p > 0, p.log() + lse[:, None] - z.gather(1, ids.long().clamp(min=0)), torch.zeros_like(p))).sum(1)
    dz = torch.exp(z - lse[:, None]).scatter_add_(1, ids.long().clamp(min=0), -p) * (2.0 / rows)
    # logits below 12, sums of 16 terms and 60000 exponentials: 2^-24 times 6 sqrt(16) 12, see above
    assert (r.lse.double() - lse).abs().max() < 3e-5 and (r.losses.double() - losses).abs().max() < 2e-4 and abs(float(r.loss) - float(losses.mean())) < 1e-4
    half, P = (2.0 ** -8, 2.0 ** -8) if dtype == "bf16" else (2.0 ** -24, 2.0 ** -14)                                # float32: exp of logits that are 5e-5 off at most
    for got, want, size in ((r.dx, dz @ W, dz.abs() @ W.abs()), (r.dw, dz.t() @ X, dz.abs().t() @ X.abs()), (r.dbias, dz.sum(0), dz.abs().sum(0))):
        assert ((got.double() - want).abs() <= (P if got is not r.dbias else 2.0 ** -13) * size + 1.01 * half * want.abs() + 1e-12).all()


def test_same_bits_every_time_and_on_another_stream():
    x, w, b, ids, top = make(13, 300, 3000, 200, "bf16", k=9)
    first = api.linear_distillation(x, w, top, ids, bias=b)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    for i in range(3):
        with torch.cuda.stream(stream):
            again = api.linear_distillation(x, w, top, ids, bias=b)
        other = api.linear_distillation(x, w, top, ids, bias=b)      # at the same time
        torch.cuda.synchronize()
        for u, v, q in zip(first, again, other):
            assert torch.equal(u, v) and torch.equal(u, q)


def test_captured_and_replayed():
    x, w, b, y, _ = make(17, 200, 1000, 96, "bf16")
    api.linear_cross_entropy(x, w, y, bias=b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = api.linear_cross_entropy(x, w, y, bias=b)
    for i in range(4):
        x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(i)).to(x))
        y.copy_(torch.randint(-1, 1000, y.shape, generator=torch.Generator().manual_seed(i)).to(y))
        graph.replay()
        eager = api.linear_cross_entropy(x, w, y, bias=b)
        torch.cuda.synchronize()
        for u, v in zip(r, eager):
            assert torch.equal(u, v), i


def test_binding_refuses():
    x, w, b, ids, top = make(1, 4, 30, 24, "bf16", k=3)
    y = ids[:, 0].contiguous()
    for bad in (lambda: api.linear_cross_entropy(x.cpu(), w, y), lambda: api.linear_cross_entropy(x, w.float(), y), lambda: api.linear_cross_entropy(x, w[:, :20], y),
                lambda: api.linear_cross_entropy(x, w, y[:3].contiguous()), lambda: api.linear_cross_entropy(x, w, y.float()), lambda: api.linear_cross_entropy(x, w, ids[:, 0]),
                lambda: api.linear_cross_entropy(x, w, y, bias=b[:20]), lambda: api.linear_cross_entropy(x, w, y, bias=b.bfloat16()), lambda: api.linear_cross_entropy(x.half(), w.half(), y),
                lambda: api.linear_cross_entropy(x.t(), w, y), lambda: api.linear_cross_entropy(x, w, y, dtype=5), lambda: api.linear_distillation(x, w, top[:, :2], ids),
                lambda: api.linear_distillation(x, w, top[:3], ids[:3]), lambda: api.linear_distillation(x, w, top.cpu(), ids), lambda: api.linear_distillation(x, w, top.half(), ids)):
        with pytest.raises(AssertionError):
            bad()
    with pytest.raises(api.SlpError):
        api.linear_distillation(x, w, top, ids, temperature=0.0)
    with pytest.raises(api.SlpError):
        api.linear_distillation(x, w, top[:, :0], ids[:, :0])
    with pytest.raises(api.SlpError):
        api.linear_cross_entropy(x[:, :0], w[:, :0], y)
