"""Performance cases of a last layer over many classes: what a program that trains it, distils into it or serves it has the framework do.

Three operators, through the public binding (paper_2403_11204_amd.api) or, for comparison, in elementary torch operations:

  xent      softmax cross-entropy over the classes of a linear layer, logits z = x W^T + b that are never kept as a whole: the mean loss over the
            rows that have a class, each row's loss and log-sum-exp, and the gradients of x, W and b
  distil    the same against a teacher's top logits: p = softmax(top / T) over each row's entries, loss T^2 KL(p || softmax(z / T)), T^2 times
            the mean's gradient
  integers  a layer in 8-bit integers: the rows of x to integers with a scale for each row, their product with weights that have a scale for each
            output channel, bias and ReLU

A class id outside [0, classes) is no class: a row without one, or without any entry of the teacher's, counts neither in the mean nor in a gradient.
An 8-bit integer matrix holds round(127 x / max|x|) of each row, ties to even, and max|x| / 127 as the row's scale.
"""

import math

import torch

own = False

DEV = "cuda"
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one row's loss over a large set of classes: scoring a single sample, bound by reading the weights once
        {"name": "xent_score_row", "kind": "xent", "rows": 1, "classes": 131072, "dim": 4096, "dtype": "bf16", "bias": False, "gradients": "none"},
        # a small last layer on a small batch: latency
        {"name": "xent_small", "kind": "xent", "rows": 64, "classes": 1000, "dim": 512, "dtype": "fp32", "bias": True, "gradients": "all"},
        # a user's own network, sizes that divide by nothing, float32
        {"name": "xent_ragged", "kind": "xent", "rows": 333, "classes": 5001, "dim": 777, "dtype": "fp32", "bias": True, "gradients": "all"},
        # a large vocabulary on a short batch
        {"name": "xent_batch", "kind": "xent", "rows": 2048, "classes": 32000, "dim": 4096, "dtype": "bf16", "bias": True, "gradients": "all"},
        # the largest: a training step's last layer, as wide as the wide configuration, on the comparison configuration's batch
        {"name": "xent_large", "kind": "xent", "rows": 8192, "classes": 131072, "dim": 4096, "dtype": "bf16", "bias": False, "gradients": "all"},
        # a teacher's eight best classes on a small batch: latency
        {"name": "distil_small", "kind": "distil", "rows": 64, "classes": 1000, "dim": 512, "dtype": "bf16", "bias": True, "gradients": "all", "top": 8,
         "temperature": 1.0},
        # a user's own network, odd sizes, entries and rows left out, a frozen last layer: only the gradient that goes on below it
        {"name": "distil_frozen_ragged", "kind": "distil", "rows": 1000, "classes": 50001, "dim": 1500, "dtype": "bf16", "bias": True,
         "gradients": "input", "top": 17, "temperature": 2.0},
        # a training step from a teacher's 64 best classes
        {"name": "distil_large", "kind": "distil", "rows": 4096, "classes": 65536, "dim": 4096, "dtype": "bf16", "bias": False, "gradients": "all",
         "top": 64, "temperature": 2.0},
        # one row through a layer of the wide configuration: bound by reading the weights once
        {"name": "integers_token", "kind": "integers", "m": 1, "n": 4096, "k": 4096, "dtype": "bf16", "bias": True, "relu": True},
        # a request of several rows
        {"name": "integers_rows", "kind": "integers", "m": 48, "n": 4096, "k": 8192, "dtype": "bf16", "bias": False, "relu": False},
        # a layer of a user's own network on its batch, float32
        {"name": "integers_ragged", "kind": "integers", "m": 1000, "n": 3001, "k": 1500, "dtype": "fp32", "bias": True, "relu": False},
        # a hidden layer of the comparison configuration
        {"name": "integers_wide", "kind": "integers", "m": 8192, "n": 16384, "k": 16384, "dtype": "bf16", "bias": True, "relu": True},
    ]


# ---- drawn cases ------------------------------------------------------------------------------------------------
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    w = _log(rng, lo, hi)
    if rng.random() < 0.5:                     # half of the widths in use are powers of two
        w = 1 << round(math.log2(w))
    return max(lo, min(hi, w))


def draw(rng):
    """One more case of the ranges that the listed ones stand for."""
    kind = rng.choice(["xent", "distil", "integers"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    if kind == "integers":
        return {"kind": kind, "m": _log(rng, 1, 8192), "n": _width(rng, 16, 16384), "k": _width(rng, 16, 16384), "dtype": dtype,
                "bias": rng.random() < 0.6, "relu": rng.random() < 0.5}
    case = {"kind": kind, "rows": _log(rng, 1, 8192), "classes": _width(rng, 16, 131072), "dim": _width(rng, 16, 8192), "dtype": dtype,
            "bias": rng.random() < 0.6, "gradients": rng.choice(["all", "all", "all", "input", "none"])}
    while case["rows"] * case["classes"] * case["dim"] > (1 << 41 if dtype == "bf16" else 1 << 38):
        side = max(("classes", "dim"), key=lambda s: case[s])
        case[side] = (case[side] + 1) // 2
    if kind == "distil":
        case["top"] = min(_log(rng, 1, 128), case["classes"])
        case["temperature"] = rng.choice([1.0, 2.0, 4.0])
    return case


# ---- a case's data ----------------------------------------------------------------------------------------------
def _integers(x):
    """(integers, scale of each row) of a float32 matrix.  The quotients in 64 bits: some lie next to a half."""
    amax = x.abs().amax(1)
    q = torch.empty(x.shape, dtype=torch.int8, device=x.device)
    for i in range(0, x.shape[0], 2048):
        a = amax[i:i + 2048, None].double()
        q[i:i + 2048] = (x[i:i + 2048].double() * 127 / torch.where(a > 0, a, torch.ones_like(a))).round().to(torch.int8)
    return q, amax / 127


def _rows128(q):
    """A matrix of bytes with rows on 128-byte boundaries and not a multiple of 4 KB apart, as the framework lays it out."""
    r, c = q.shape
    ld = -(-c // 128) * 128
    ld += 128 if ld % 4096 == 0 else 0
    full = torch.zeros(r, ld, dtype=q.dtype, device=q.device)
    full[:, :c] = q
    return full[:, :c]


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    s = {"case": case}
    if case["kind"] == "integers":
        m, n, k = case["m"], case["n"], case["k"]
        x = torch.randn(m, k, device=DEV, generator=gen)
        s["x"] = x.mul_(torch.randn(m, 1, device=DEV, generator=gen).exp_()).to(dt)
        w = torch.randn(n, k, device=DEV, generator=gen).div_(math.sqrt(k))
        q, scale = _integers(w)
        s["w"] = (_rows128(q), scale)
        s["bias"] = torch.randn(n, device=DEV, generator=gen).mul_(0.1) if case["bias"] else None
        return s
    r, c, d = case["rows"], case["classes"], case["dim"]
    s["x"] = torch.randn(r, d, device=DEV, generator=gen).to(dt)
    w = torch.randn(c, d, device=DEV, generator=gen).mul_(2.5 / math.sqrt(d))      # logits as spread as a partly trained layer's
    s["w"] = w.to(dt)
    s["bias"] = torch.randn(c, device=DEV, generator=gen).mul_(0.1) if case["bias"] else None
    if case["kind"] == "xent":
        y = torch.randint(c, (r,), device=DEV, generator=gen, dtype=torch.int32)
        s["y"] = torch.where(torch.rand(r, device=DEV, generator=gen) < (0.1 if r > 1 else 0.0), -1, y).int()    # rows without a class: padding
        return s
    # a teacher that agrees with the student in part: its top logits, best first, some lists shorter than others and some rows without one
    k = case["top"]
    top = torch.empty(r, k, device=DEV)
    ids = torch.empty(r, k, dtype=torch.int64, device=DEV)
    for i in range(0, r, 1024):
        z = torch.mm(s["x"][i:i + 1024].to(torch.bfloat16), s["w"].to(torch.bfloat16).t()).float()
        z += 1.5 * torch.randn(z.shape, device=DEV, generator=gen)
        top[i:i + 1024], ids[i:i + 1024] = z.topk(k, 1)
    length = torch.randint(1, k + 1, (r, 1), device=DEV, generator=gen)
    length = torch.where(torch.rand(r, 1, device=DEV, generator=gen) < 0.7, torch.full_like(length, k), length)
    if r > 1:
        length = torch.where(torch.rand(r, 1, device=DEV, generator=gen) < 0.05, torch.zeros_like(length), length)
    s["top"] = top.to(dt)
    s["ids"] = torch.where(torch.arange(k, device=DEV) < length, ids, torch.full_like(ids, -1)).int()
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------
def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    from paper_2403_11204_amd import api

    case = s["case"]
    if case["kind"] == "integers":
        x8 = api.quantize_integers(s["x"])
        return api.product_integers(x8, api.Integers(*s["w"]), bias=s["bias"], relu=case["relu"], dtype=api.BF16 if case["dtype"] == "bf16" else api.F32)
    grads = {"gradients": case["gradients"] != "none", "weight_gradients": case["gradients"] == "all"}
    if case["kind"] == "xent":
        r = api.linear_cross_entropy(s["x"], s["w"], s["y"], bias=s["bias"], **grads)
    else:
        r = api.linear_distillation(s["x"], s["w"], s["top"], s["ids"], bias=s["bias"], temperature=case["temperature"], **grads)
    out = {"loss": r.loss, "losses": r.losses, "lse": r.lse}
    if case["gradients"] != "none":
        out["dx"] = r.dx
    if case["gradients"] == "all":
        out["dw"] = r.dw
        if case["bias"]:
            out["dbias"] = r.dbias
    return out


def _plain(s):
    case = s["case"]
    if case["kind"] == "integers":
        q, scale = _integers(s["x"].float())
        wq, wscale = s["w"]
        out = (q.float() @ wq.float().t()) * scale[:, None] * wscale
        if s["bias"] is not None:
            out = out + s["bias"]
        if case["relu"]:
            out = out.clamp(min=0)
        return out.to(s["x"].dtype)
    x, w = s["x"].float(), s["w"].float()
    temperature = case["temperature"] if case["kind"] == "distil" else 1.0
    z = x @ w.t()
    if s["bias"] is not None:
        z += s["bias"]
    if temperature != 1.0:
        z /= temperature
    peak = z.amax(1, keepdim=True)
    lse = (z - peak).exp().sum(1).log() + peak[:, 0]
    if case["kind"] == "xent":
        ids = s["y"].long()[:, None]
        given = ids >= 0
        p = given.float()
        entropy = 0.0
    else:
        ids = s["ids"].long()
        given = ids >= 0
        t = s["top"].float() / temperature
        t = torch.where(given, t, torch.full_like(t, -math.inf))
        best = t.amax(1, keepdim=True)
        e = torch.where(given, (t - torch.where(best > -math.inf, best, torch.zeros_like(best))).exp(), torch.zeros_like(t))
        p = e / e.sum(1, keepdim=True).clamp(min=1e-30)
        entropy = torch.where(p > 0, p * p.clamp(min=1e-38).log(), torch.zeros_like(p)).sum(1)
    counts = given.any(1)
    at = ids.clamp(min=0)
    square = temperature * temperature
    losses = (entropy + lse * p.sum(1) - (p * z.gather(1, at)).sum(1)) * square * counts
    n = counts.sum().clamp(min=1).float()
    out = {"loss": losses.sum() / n, "losses": losses, "lse": lse}
    if case["gradients"] == "none":
        return out
    g = z.sub_(lse[:, None]).exp_()
    g.scatter_add_(1, at, -p)
    g *= (counts.float() * temperature / n)[:, None]
    out["dx"] = (g @ w).to(s["x"].dtype)
    if case["gradients"] == "all":
        out["dw"] = (g.t() @ x).to(s["w"].dtype)
        if s["bias"] is not None:
            out["dbias"] = g.sum(0)
    return out


# ---- what a pass cannot do without ------------------------------------------------------------------------------
def work(case):
    es = DTYPES[case["dtype"]].itemsize
    if case["kind"] == "integers":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": m * k * es + n * k + 4 * n + m * n * es, "flops": 2 * m * n * k}
    r, c, d = case["rows"], case["classes"], case["dim"]
    products = {"none": 1, "input": 2, "all": 3}[case["gradients"]]
    sides = es * (r * d * (2 if products > 1 else 1) + c * d * (2 if products > 2 else 1))
    entries = r * case["top"] * (es + 4) if case["kind"] == "distil" else 4 * r
    return {"bytes": sides + entries + 8 * r + (8 * c if case["bias"] and products > 2 else 4 * c if case["bias"] else 0), "flops": 2 * products * r * c * d}


# ---- the same in 64 bits, from the definitions -------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "integers":
        x = s["x"].double()
        largest = x.abs().max(dim=1, keepdim=True).values
        unit = torch.where(largest > 0, largest, torch.ones_like(largest)) / 127
        whole = torch.round(127 * x / torch.where(largest > 0, largest, torch.ones_like(largest)))
        out = torch.mm(whole * torch.where(largest > 0, unit, torch.zeros_like(unit)), (s["w"][0].double() * s["w"][1].double().unsqueeze(1)).t().contiguous())
        if s["bias"] is not None:
            out += s["bias"].double()
        return torch.where(out > 0, out, torch.zeros_like(out)) if case["relu"] else out
    # L_i = T^2 sum_j p_ij (log p_ij - log q_i,c(j)), q_i = softmax(z_i / T);  dL_i / dz_iv = T (q_iv - sum of p_ij with c(j) = v)
    big_t = case["temperature"] if case["kind"] == "distil" else 1.0
    x, w = s["x"].double(), s["w"].double()
    logq = torch.mm(x, w.t().contiguous())
    if s["bias"] is not None:
        logq += s["bias"].double()
    logq /= big_t
    lse = torch.logsumexp(logq, 1)
    logq -= lse.unsqueeze(1)
    rows = torch.arange(case["rows"], device=DEV)
    if case["kind"] == "xent":
        columns = [(s["y"].long(), torch.ones(case["rows"], dtype=torch.float64, device=DEV))]
        any_given = s["y"] >= 0
    else:
        t = s["top"].double() / big_t
        t = t.masked_fill(s["ids"] < 0, -math.inf)
        any_given = (s["ids"] >= 0).sum(1) > 0
        p = torch.softmax(torch.where(any_given.unsqueeze(1), t, torch.zeros_like(t)), 1)
        columns = [(s["ids"][:, j].long(), p[:, j]) for j in range(case["top"])]
    losses = torch.zeros(case["rows"], dtype=torch.float64, device=DEV)
    for c, p in columns:
        use = (c >= 0) & (p > 0)
        losses[use] += p[use] * (torch.log(p[use]) - logq[rows[use], c[use]])
    losses *= big_t ** 2
    n = max(1, int(any_given.sum()))
    out = {"loss": losses.sum() / n, "losses": losses, "lse": lse}
    if case["gradients"] == "none":
        return out
    dz = logq.exp_()
    for c, p in columns:
        use = c >= 0
        dz[rows[use], c[use]] -= p[use]
    dz *= (any_given.double() * (big_t / n)).unsqueeze(1)
    out["dx"] = torch.mm(dz, w)
    if case["gradients"] == "all":
        out["dw"] = torch.mm(dz.t().contiguous(), x)
        if s["bias"] is not None:
            out["dbias"] = dz.sum(0)
    return out
