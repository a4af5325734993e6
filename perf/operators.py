"""Performance cases of the 8-bit operators: what a program that trains or serves segments in 8 bits has the framework do.

Four operators, through the public binding (paper_2403_11204_amd.api) or, for comparison, in elementary torch operations:

  norm, norm_back   root-mean-square norm with the residual's addition and an output in 8 bits with a scale for each 128
                    elements of a row; its backward pass
  quantize          a matrix to 8 bits, one scale for each 128 elements of a row or for each 128 x 128 block, row-major,
                    transposed or both, with the ReLU mask and the column sums of a gradient
  product, layer_back   the product of two such matrices with bias and ReLU; the backward pass of a layer (the gradient of its
                    output to 8 bits in both layouts, the gradients of its input, weights and bias)
  clip              the norm of all gradients of a segment together, and the gradients scaled to a given norm

8-bit values are e4m3, scales are powers of two (e8m0), both in torch's types for them.  The scale of a block is the least
power of two 2^e, e >= -127, with max|x| <= 448 2^e.
"""

import math

import torch

own = False

DEV = "cuda"
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
EPS = 1e-6


def _dash(widths):
    return "-".join(str(w) for w in widths)


def listed():
    return [
        # one row through a residual segment as wide as the wide configuration: what serving a single sample asks for
        {"name": "norm_token", "kind": "norm", "rows": 1, "dim": 4096, "dtype": "bf16", "residual": True},
        # a batch of the comparison configuration, the largest norm
        {"name": "norm_wide", "kind": "norm", "rows": 8192, "dim": 16384, "dtype": "bf16", "residual": True},
        # the backward pass at the deep configuration's batch and width
        {"name": "norm_back_deep", "kind": "norm_back", "rows": 4096, "dim": 8192, "dtype": "bf16", "residual": True},
        # the weights of one layer of the deep configuration after an update, for the forward product and the data gradient
        {"name": "quantize_weights", "kind": "quantize", "rows": 8192, "cols": 8192, "dtype": "fp32", "block": 128,
         "layouts": "both", "masked": False},
        # a gradient of a user's own network, sizes that divide by nothing, float32, for both backward products
        {"name": "quantize_ragged", "kind": "quantize", "rows": 1000, "cols": 3001, "dtype": "fp32", "block": 1,
         "layouts": "both", "masked": True},
        # one row through a layer of the wide configuration: bound by reading the weights once
        {"name": "product_token", "kind": "product", "m": 1, "n": 4096, "k": 4096, "out": "bf16", "bias": True, "relu": True},
        # a layer of a user's own network on its batch
        {"name": "product_ragged", "kind": "product", "m": 1000, "n": 3001, "k": 1500, "out": "fp32", "bias": True, "relu": False},
        # a hidden layer of the comparison configuration, the largest product
        {"name": "product_wide", "kind": "product", "m": 8192, "n": 16384, "k": 16384, "out": "bf16", "bias": True, "relu": True},
        # the backward pass of a user's own layer on a short last batch
        {"name": "layer_back_ragged", "kind": "layer_back", "m": 333, "n": 777, "k": 3001, "dtype": "fp32"},
        # the backward pass of a layer of the deep configuration on its batch
        {"name": "layer_back_deep", "kind": "layer_back", "m": 4096, "n": 8192, "k": 8192, "dtype": "bf16"},
        # the gradients of the left partition of the network of the paper's experiment: latency
        {"name": "clip_paper", "kind": "clip", "widths": "784-80-60", "dtype": "fp32", "share": 0.5},
        # the gradients of the left segment of the comparison configuration: every one of 549 million values
        {"name": "clip_comparison", "kind": "clip", "widths": "784-16384-16384-16384", "dtype": "fp32", "share": 0.5},
    ]


# ---- drawn cases ------------------------------------------------------------------------------------------------
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    w = _log(rng, lo, hi)
    if rng.random() < 0.5:                     # half of the widths in use are powers of two
        w = 1 << round(math.log2(w))
    return max(lo, min(hi, w))


def _parameters(widths):
    return sum((a + 1) * b for a, b in zip(widths, widths[1:]))


def draw(rng):
    """One more case of the ranges that the listed ones stand for."""
    kind = rng.choice(["norm", "norm_back", "quantize", "product", "product", "layer_back", "clip"])
    dtype = rng.choice(["bf16", "fp32"])
    if kind in ("norm", "norm_back"):
        dim = _width(rng, 16, 16384)
        return {"kind": kind, "rows": _log(rng, 1, 8192), "dim": dim, "dtype": dtype, "residual": rng.random() < 0.7}
    if kind == "quantize":
        block = rng.choice([1, 128])
        return {"kind": kind, "rows": _log(rng, 1, 8192), "cols": _width(rng, 16, 16384), "dtype": dtype, "block": block,
                "layouts": rng.choice(["rows", "transposed", "both"]), "masked": block == 1 and rng.random() < 0.5}
    if kind == "product":
        return {"kind": kind, "m": _log(rng, 1, 8192), "n": _width(rng, 16, 16384), "k": _width(rng, 16, 16384),
                "out": rng.choice(["bf16", "fp32"]), "bias": rng.random() < 0.7, "relu": rng.random() < 0.5}
    if kind == "layer_back":
        return {"kind": kind, "m": _log(rng, 1, 4096), "n": _width(rng, 16, 8192), "k": _width(rng, 16, 8192), "dtype": dtype}
    widths = [_width(rng, 16, 16384) for _ in range(rng.randint(2, 13))]
    while _parameters(widths) > 500_000_000:
        widths[widths.index(max(widths))] //= 2
    return {"kind": kind, "widths": _dash(widths), "dtype": dtype, "share": rng.choice([0.5, 2.0])}


# ---- 8-bit matrices in elementary operations --------------------------------------------------------------------
def _spread(x, rows, cols):
    """The block scales, one for each `rows` x `cols` elements of a matrix whose sides they divide, as the matrix's elements see them."""
    return x.repeat_interleave(rows, 0).repeat_interleave(cols, 1)


def _quantize(x, block):
    """(values in e4m3, scales in e8m0) of a float32 matrix: a scale for each `block` rows x 128 columns."""
    r, c = x.shape
    x = torch.nn.functional.pad(x, (0, -c % 128, 0, -r % block))
    amax = x.abs().reshape(x.shape[0] // block, block, x.shape[1] // 128, 128).amax((1, 3))
    m, e = torch.frexp(amax)                                   # amax = m 2^e, m in [0.5, 1); 448 = 0.875 2^9
    e = torch.where(amax > 0, e - 9 + (m > 0.875).int(), -127).clamp(min=-127)
    up = ((127 - e.int()) << 23).view(torch.float32)           # 2^-e
    q = (x * _spread(up, block, 128))[:r, :c].to(E4M3)
    return q, (e + 127).to(torch.uint8).view(E8M0)


def _dequantize(q, scales, block):
    r, c = q.shape
    s = _spread(scales.float(), block, 128)[:r, :c]
    return q.float() * s


# ---- a case's data ----------------------------------------------------------------------------------------------
def _values(gen, rows, cols, dtype):
    """Activations or gradients: normal, the size of a row spread over a factor of a few."""
    x = torch.randn(rows, cols, device=DEV, generator=gen)
    return x.mul_(torch.randn(rows, 1, device=DEV, generator=gen).exp_()).to(dtype)


def _rows8(q, scales):
    """An 8-bit matrix laid out as the framework lays it out: rows on 128-byte boundaries and not a multiple of 4 KB apart, pads zero; rows of
    scales on 4-byte boundaries."""
    r, c = q.shape
    ld = -(-c // 128) * 128
    ld += 128 if ld % 4096 == 0 else 0
    full = torch.zeros(r, ld, dtype=torch.uint8, device=q.device)
    full[:, :c] = q.view(torch.uint8)
    sr, sc = scales.shape
    sfull = torch.zeros(sr, -(-sc // 4) * 4, dtype=torch.uint8, device=q.device)
    sfull[:, :sc] = scales.view(torch.uint8)
    return full.view(E4M3)[:, :c], sfull.view(E8M0)[:, :sc]


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    kind = case["kind"]
    s = {"case": case}
    if kind in ("norm", "norm_back"):
        dt = DTYPES[case["dtype"]]
        rows, dim = case["rows"], case["dim"]
        s["gamma"] = 1 + 0.1 * torch.randn(dim, device=DEV, generator=gen)
        s["x"] = _values(gen, rows, dim, dt)
        s["residual"] = _values(gen, rows, dim, dt) if case["residual"] else None
        if kind == "norm_back":              # what the forward pass left
            s["dy"] = _values(gen, rows, dim, dt).mul_(1e-3)
            s["residual"] = s["residual"].mul_(1e-3) if case["residual"] else None     # the gradient that reaches the sum past the norm
            s["rstd"] = torch.rsqrt(s["x"].float().square().mean(1) + EPS)
    elif kind == "quantize":
        dt = DTYPES[case["dtype"]]
        s["x"] = _values(gen, case["rows"], case["cols"], dt).mul_(1e-3)
        s["mask"] = torch.randn(case["rows"], case["cols"], device=DEV, generator=gen).clamp_(min=0).to(dt) if case["masked"] else None
    elif kind in ("product", "layer_back"):
        m, n, k = case["m"], case["n"], case["k"]
        w = torch.randn(n, k, device=DEV, generator=gen).div_(math.sqrt(k))
        x = _values(gen, m, k, torch.float32)
        if kind == "product":
            s["x8"], s["w8"] = _rows8(*_quantize(x, 1)), _rows8(*_quantize(w, 128))
            s["bias"] = torch.randn(n, device=DEV, generator=gen).mul_(0.1) if case["bias"] else None
        else:                                # the layer's weights and input, transposed, as the forward pass kept them
            dt = DTYPES[case["dtype"]]
            s["xt8"], s["wt8"] = _rows8(*_quantize(x.t().contiguous(), 1)), _rows8(*_quantize(w.t().contiguous(), 128))
            s["da"] = _values(gen, m, n, dt).mul_(1e-3)
            s["a"] = torch.randn(m, n, device=DEV, generator=gen).clamp_(min=0).to(dt)
    else:
        widths = [int(w) for w in case["widths"].split("-")]
        dt = DTYPES[case["dtype"]]
        shapes = [shape for a, b in zip(widths, widths[1:]) for shape in ((b, a), (b,))]
        s["grads"] = [torch.randn(shape, device=DEV, generator=gen).mul_(1e-3).to(dt) for shape in shapes]
        s["out"] = [torch.empty_like(g) for g in s["grads"]]
        s["max_norm"] = case["share"] * 1e-3 * math.sqrt(_parameters(widths))
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------
def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    from paper_2403_11204_amd import api

    case = s["case"]
    kind = case["kind"]
    if kind == "norm":
        n = api.rmsnorm(s["x"], s["gamma"], residual=s["residual"], eps=EPS)
        return {"h": n.h, "rstd": n.rstd, "q": n.y8.q, "scales": n.y8.scales}
    if kind == "norm_back":
        dx, dgamma = api.rmsnorm_backward(s["dy"], s["x"], s["gamma"], s["rstd"], dh=s["residual"])
        return {"dx": dx, "dgamma": dgamma}
    if kind == "quantize":
        lay = case["layouts"]
        r = api.quantize(s["x"], block=case["block"], rows=lay != "transposed", transposed=lay != "rows", mask=s["mask"], column_sums=case["masked"])
        out = {}
        if r.rows is not None:
            out |= {"q": r.rows.q, "scales": r.rows.scales}
        if r.transposed is not None:
            out |= {"qt": r.transposed.q, "scales_t": r.transposed.scales}
        if r.column_sums is not None:
            out["sums"] = r.column_sums
        return out
    if kind == "product":
        return api.product(api.Quantized(*s["x8"], 1), api.Quantized(*s["w8"], 128), bias=s["bias"], relu=case["relu"],
                           dtype=api.BF16 if case["out"] == "bf16" else api.F32)
    if kind == "layer_back":
        dz = api.quantize(s["da"], rows=True, transposed=True, mask=s["a"], column_sums=True)
        dx = api.product(dz.rows, api.Quantized(*s["wt8"], 128), dtype=api.BF16 if case["dtype"] == "bf16" else api.F32)
        dw = api.product(dz.transposed, api.Quantized(*s["xt8"], 1), dtype=api.F32)
        return {"dx": dx, "dw": dw, "db": dz.column_sums}
    norm = api.clip_gradients(s["grads"], s["max_norm"], out=s["out"])
    return {"norm": norm, "grads": s["out"]}


def _plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "norm":
        x = s["x"].float()
        if s["residual"] is not None:
            x = x + s["residual"].float()
        h = x.to(s["x"].dtype)               # the norm is of what is stored
        hf = h.float()
        rstd = 1 / torch.sqrt((hf * hf).mean(1) + EPS)
        q, scales = _quantize(hf * rstd[:, None] * s["gamma"], 1)
        return {"h": h, "rstd": rstd, "q": q, "scales": scales}
    if kind == "norm_back":
        h, dy, rstd = s["x"].float(), s["dy"].float(), s["rstd"][:, None]
        g = dy * s["gamma"]
        dx = rstd * (g - h * (rstd * rstd * (g * h).mean(1, keepdim=True)))
        if s["residual"] is not None:
            dx = dx + s["residual"].float()
        return {"dx": dx.to(s["x"].dtype), "dgamma": (dy * h * rstd).sum(0)}
    if kind == "quantize":
        x = s["x"].float()
        if s["mask"] is not None:
            x = x * (s["mask"] > 0)
        out = {}
        if case["layouts"] != "transposed":
            out["q"], out["scales"] = _quantize(x, case["block"])
        if case["layouts"] != "rows":
            out["qt"], out["scales_t"] = _quantize(x.t().contiguous(), case["block"])
        if case["masked"]:
            out["sums"] = x.sum(0)
        return out
    if kind == "product":
        out = _dequantize(*s["x8"], 1) @ _dequantize(*s["w8"], 128).t()
        if s["bias"] is not None:
            out = out + s["bias"]
        if case["relu"]:
            out = out.clamp(min=0)
        return out.to(DTYPES[case["out"]])
    if kind == "layer_back":
        dz = s["da"].float() * (s["a"] > 0)
        dx = _dequantize(*_quantize(dz, 1), 1) @ _dequantize(*s["wt8"], 128).t()
        dw = _dequantize(*_quantize(dz.t().contiguous(), 1), 1) @ _dequantize(*s["xt8"], 1).t()
        return {"dx": dx.to(s["da"].dtype), "dw": dw, "db": dz.sum(0)}
    grads = [g.float() for g in s["grads"]]
    norm = torch.sqrt(torch.stack([(g * g).sum() for g in grads]).sum())
    c = (s["max_norm"] / (norm + 1e-6)).clamp(max=1)
    return {"norm": norm, "grads": [(g * c).to(DTYPES[case["dtype"]]) for g in grads]}


# ---- what a pass cannot do without ------------------------------------------------------------------------------
def work(case):
    kind = case["kind"]
    blocks = lambda n: -(-n // 128)  # noqa: E731
    if kind == "norm":
        r, d, es = case["rows"], case["dim"], DTYPES[case["dtype"]].itemsize
        return {"bytes": r * d * (es * (3 if case["residual"] else 1) + 1) + r * (blocks(d) + 4) + 4 * d, "flops": 6 * r * d}
    if kind == "norm_back":
        r, d, es = case["rows"], case["dim"], DTYPES[case["dtype"]].itemsize
        return {"bytes": r * d * es * (4 if case["residual"] else 3) + 4 * r + 8 * d, "flops": 10 * r * d}
    if kind == "quantize":
        r, c, es = case["rows"], case["cols"], DTYPES[case["dtype"]].itemsize
        return {"bytes": r * c * (es * (2 if case["masked"] else 1) + (2 if case["layouts"] == "both" else 1)), "flops": 3 * r * c}
    if kind == "product":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": (m + n) * k + m * n * DTYPES[case["out"]].itemsize, "flops": 2 * m * n * k}
    if kind == "layer_back":
        m, n, k, es = case["m"], case["n"], case["k"], DTYPES[case["dtype"]].itemsize
        return {"bytes": 2 * es * m * n + (m + n) * k + es * m * k + 4 * n * k, "flops": 4 * m * n * k}
    p = _parameters([int(w) for w in case["widths"].split("-")])
    return {"bytes": 2 * p * DTYPES[case["dtype"]].itemsize, "flops": 3 * p}


# ---- the same in 64 bits, from the definitions -------------------------------------------------------------------
def _exponents64(x, block):
    """e of every block's scale 2^e, the least one >= -127 with max|x| <= 448 2^e."""
    r, c = x.shape
    rows, cols = -(-r // block), -(-c // 128)
    full = x.new_zeros(rows * block, cols * 128)
    full[:r, :c] = x.abs()
    amax = full.view(rows, block, cols, 128).amax(3).amax(1)
    e = torch.log2(amax / 448).ceil().clamp(min=-130, max=130)
    e = torch.where(amax <= 448 * torch.exp2(e - 1), e - 1, e)     # log2 may have rounded across a power of two
    e = torch.where(amax > 448 * torch.exp2(e), e + 1, e)
    return torch.where(amax > 0, e, torch.full_like(e, -127)).clamp(min=-127)


def _elements64(e, block, shape):
    i = torch.arange(shape[0], device=e.device) // block
    j = torch.arange(shape[1], device=e.device) // 128
    return torch.exp2(e)[i][:, j]


def _round64(v):
    """To the nearest e4m3 value, ties to the even one: 3 bits behind the leading one, steps of 2^-9 below 2^-6."""
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(v / step) * step


def _quantized64(x, block):
    s = _elements64(_exponents64(x, block), block, x.shape)
    return _round64(x / s) * s


def _scaled64(x, block):
    """What the 8-bit values stand for before they are rounded, and the scales."""
    e = _exponents64(x, block)
    return x / _elements64(e, block, x.shape), torch.exp2(e)


def _value64(matrix, block):
    q, scales = matrix
    return q.float().double() * _elements64(torch.log2(scales.float().double()).round(), block, q.shape)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "norm":
        x = s["x"].double()
        if s["residual"] is not None:
            x = x + s["residual"].double()
        stored = x.to(s["x"].dtype).double()
        rstd = (stored.pow(2).sum(1) / case["dim"] + EPS).pow(-0.5)
        q, scales = _scaled64(stored * rstd.unsqueeze(1) * s["gamma"].double(), 1)
        return {"h": x, "rstd": rstd, "q": q, "scales": scales}
    if kind == "norm_back":
        # y_i = gamma_i h_i n(h): dx_j = sum_i dy_i gamma_i (n [i = j] - h_i n^3 h_j / dim)
        h, dy, n, gamma = s["x"].double(), s["dy"].double(), s["rstd"].double().unsqueeze(1), s["gamma"].double()
        along = ((dy * gamma * h).sum(1) / case["dim"]).unsqueeze(1)
        dx = dy * gamma * n - h * along * n.pow(3)
        if s["residual"] is not None:
            dx = dx + s["residual"].double()
        return {"dx": dx, "dgamma": (dy * h * n).sum(0)}
    if kind == "quantize":
        x = s["x"].double()
        if s["mask"] is not None:
            x = torch.where(s["mask"] > 0, x, torch.zeros_like(x))
        out = {}
        if case["layouts"] != "transposed":
            out["q"], out["scales"] = _scaled64(x, case["block"])
        if case["layouts"] != "rows":
            out["qt"], out["scales_t"] = _scaled64(x.t(), case["block"])
        if case["masked"]:
            out["sums"] = x.sum(0)
        return out
    if kind == "product":
        out = torch.mm(_value64(s["x8"], 1), _value64(s["w8"], 128).t().contiguous())
        if s["bias"] is not None:
            out += s["bias"].double()
        return torch.where(out > 0, out, torch.zeros_like(out)) if case["relu"] else out
    if kind == "layer_back":
        dz = torch.where(s["a"] > 0, s["da"].double(), torch.zeros((), dtype=torch.float64, device=DEV))
        dx = torch.mm(_quantized64(dz, 1), _value64(s["wt8"], 128).t().contiguous())
        dw = torch.mm(_quantized64(dz.t().contiguous(), 1), _value64(s["xt8"], 1).t().contiguous())
        return {"dx": dx, "dw": dw, "db": dz.sum(0)}
    grads = [g.double() for g in s["grads"]]
    norm = sum(g.pow(2).sum() for g in grads) ** 0.5
    c = min(1.0, s["max_norm"] / (float(norm) + 1e-6))
    return {"norm": norm, "grads": [g * c for g in grads]}
