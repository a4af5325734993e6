"""Oracle of the 8-bit operators and of gradient clipping, in float64 from their definitions.

An 8-bit matrix is (q, e): q float64 holding e4m3 values (sign, 4 exponent bits with bias 7, 3 fraction bits, largest 448, steps of 2^-9 around
zero), e integer exponents, one for each `block` rows x 128 columns; it stands for q * 2^e.
"""

import numpy as np

LARGEST = 448.0


def to_e4m3(v):
    """Nearest e4m3 value of |v| <= 448, ties to an even fraction."""
    v = np.asarray(v, dtype=np.float64)
    exponent = np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -6)))
    step = 2.0 ** (exponent - 3)
    return np.rint(v / step) * step                        # (rounding up to the next power of two stays on the grid)


def bits_of(q):
    """The bytes of e4m3 values."""
    q = np.asarray(q, dtype=np.float64)
    a = np.abs(q)
    exponent = np.floor(np.log2(np.maximum(a, 2.0 ** -6)))
    fraction = np.where(a < 2.0 ** -6, a * 2.0 ** 9, (a / 2.0 ** exponent - 1) * 8)
    field = np.where(a < 2.0 ** -6, 0, exponent + 7)
    return (np.signbit(q) * 128 + field * 8 + fraction).astype(np.uint8)


def exponents(x, block):
    """The least e >= -127 with max|x| <= 448 * 2^e, for each block x 128 elements."""
    r, c = x.shape
    out = np.empty((-(-r // block), -(-c // 128)), dtype=np.int64)
    for i in range(out.shape[0]):
        for j in range(out.shape[1]):
            big = np.max(np.abs(x[i * block:(i + 1) * block, j * 128:(j + 1) * 128]), initial=0.0)
            e = -127
            if big > 0:
                e = max(-127, int(np.floor(np.log2(big / LARGEST))) - 1)
                while big > LARGEST * 2.0 ** e:
                    e += 1
            out[i, j] = e
    return out


def spread(e, block, shape):
    """The exponents as the elements see them."""
    return np.repeat(np.repeat(e, block, 0)[:shape[0]], 128, 1)[:, :shape[1]]


def quantize(x, block):
    x = np.asarray(x, dtype=np.float64)
    e = exponents(x, block)
    return to_e4m3(x / 2.0 ** spread(e, block, x.shape)), e


def dequantize(q, e, block):
    return q * 2.0 ** spread(e, block, q.shape)


def product(a, b, bias=None, relu=False):
    """act(a b^T + bias) of dequantised matrices."""
    z = a @ b.T
    if bias is not None:
        z = z + np.asarray(bias, dtype=np.float64)
    return np.maximum(z, 0.0) if relu else z


def rmsnorm(h, gamma, eps):
    """(y, rstd) of the rows of h."""
    rstd = 1.0 / np.sqrt(np.mean(h * h, axis=1) + eps)
    return h * rstd[:, None] * gamma, rstd


def rmsnorm_backward(dy, h, gamma, eps, dh=None):
    """(d loss / d h, d loss / d gamma) from d loss / d y."""
    n = 1.0 / np.sqrt(np.mean(h * h, axis=1, keepdims=True) + eps)
    g = dy * gamma
    dx = n * (g - h * n * n * np.mean(g * h, axis=1, keepdims=True))
    return dx if dh is None else dx + dh, np.sum(dy * h * n, axis=0)


def clip(tensors, max_norm):
    """(norm, scaled tensors)."""
    norm = np.sqrt(sum(np.sum(t * t) for t in tensors))
    c = min(1.0, max_norm / (norm + 1e-6)) if np.isfinite(norm) else 1.0
    return norm, [t * c for t in tensors]
