"""Values in 8 bits with a scale for each block of 128, the norm, the 8-bit affine layer and AdamW, in plain numpy.

The quantisation is fixed to the bit (fp32 quotients and products, nearest even); everything else is in fp64 from the definitions in
include/distdl.h.
"""

import numpy as np

BLOCK = 128
TINY = np.float32(2.0 ** -100)
TOP = np.float32(448.0)


def e4m3_value(code):
    """fp64 values of e4m3 bytes (1 sign, 4 exponent, 3 mantissa bits, bias 7; 0x7f and 0xff are NaN)."""
    c = np.asarray(code, np.uint8).astype(np.int64)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c & 128, -v, v)


_POSITIVE = e4m3_value(np.arange(127))


def e4m3_round(x):
    """Nearest e4m3 values of finite numbers (ties to the even code), at most 448 in magnitude."""
    x = np.asarray(x, np.float64)
    a = np.minimum(np.abs(x), 448.0)
    hi = np.searchsorted(_POSITIVE, a).clip(0, 126)
    lo = (hi - 1).clip(0)
    up, down = _POSITIVE[hi] - a, a - _POSITIVE[lo]
    code = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))
    code = np.where(_POSITIVE[hi] == a, hi, code)
    return np.copysign(_POSITIVE[code], x)


def _scale(a):
    a = np.maximum(a.astype(np.float32), TINY)
    return a / TOP, TOP / a


def quantize_rows(x):
    """x: fp32 values [nb, n] -> (values of the codes [nb, n] fp64, scales [ceil(n/128), nb] fp32)."""
    x = np.asarray(x, np.float32)
    nb, n = x.shape
    pad = np.zeros((nb, -(-n // BLOCK) * BLOCK), np.float32)
    pad[:, :n] = x
    pad = pad.reshape(nb, -1, BLOCK)
    s, inv = _scale(np.abs(pad).max(2) if nb else np.zeros(pad.shape[:2], np.float32))
    q = e4m3_round(pad * inv[:, :, None]).reshape(nb, -1)[:, :n]
    return q, np.ascontiguousarray(s.T)


def quantize_weights(w):
    """w: fp32 values [rows, cols] -> (values of the codes, scales [ceil(rows/128), ceil(cols/128)])."""
    w = np.asarray(w, np.float32)
    rows, cols = w.shape
    pad = np.zeros((-(-rows // BLOCK) * BLOCK, -(-cols // BLOCK) * BLOCK), np.float32)
    pad[:rows, :cols] = w
    blocks = pad.reshape(pad.shape[0] // BLOCK, BLOCK, pad.shape[1] // BLOCK, BLOCK)
    s, inv = _scale(np.abs(blocks).max((1, 3)))
    q = e4m3_round(blocks * inv[:, None, :, None]).reshape(pad.shape)[:rows, :cols]
    return q, s


def row_values(q, s):
    """What rows in 8 bits stand for, fp64."""
    return np.asarray(q, np.float64) * np.repeat(np.asarray(s, np.float64).T, BLOCK, axis=1)[:, :q.shape[1]]


def weight_values(q, s):
    r = np.repeat(np.asarray(s, np.float64), BLOCK, axis=0)[:q.shape[0]]
    return np.asarray(q, np.float64) * np.repeat(r, BLOCK, axis=1)[:, :q.shape[1]]


def rmsnorm_fwd(h, gamma, eps):
    """h, gamma: lists of feature blocks, fp64 -> (list of y, rstd [nb])."""
    nf = sum(b.shape[1] for b in h)
    rstd = 1.0 / np.sqrt(sum((b.astype(np.float64) ** 2).sum(1) for b in h) / nf + eps)
    return [b * rstd[:, None] * g for b, g in zip(h, gamma)], rstd


def rmsnorm_adj(dy, dres, h, gamma, rstd):
    """-> (list of dh, list of dgamma); dres: list or None."""
    nf = sum(b.shape[1] for b in h)
    r = np.asarray(rstd, np.float64)[:, None]
    hat = [b * r for b in h]
    mean = sum((g * d * x).sum(1, keepdims=True) for g, d, x in zip(gamma, dy, hat)) / nf
    dh = [r * (g * d - x * mean) for g, d, x in zip(gamma, dy, hat)]
    if dres is not None:
        dh = [a + b for a, b in zip(dh, dres)]
    return dh, [(d * x).sum(0) for d, x in zip(dy, hat)]


def affine_fp8_fwd(x, w, pfo, pfi, bias=None):
    """x[j], w[i*pfi+j]: (values, scales) pairs as the quantisations give them -> list of y."""
    xv = [row_values(*a) for a in x]
    y = [sum(xv[j] @ weight_values(*w[i * pfi + j]).T for j in range(pfi)) for i in range(pfo)]
    return y if bias is None else [a + b for a, b in zip(y, bias)]


def affine_fp8_adj(dy, w, pfo, pfi):
    dv = [row_values(*a) for a in dy]
    return [sum(dv[i] @ weight_values(*w[i * pfi + j]) for i in range(pfo)) for j in range(pfi)]


MASK = np.uint64(0xFFFFFFFF)


def _mixed(x):
    x = x ^ (x >> np.uint64(16))
    x = (x * np.uint64(0xB504F333)) & MASK
    x = x ^ (x >> np.uint64(15))
    x = (x * np.uint64(0x93CD3A2D)) & MASK
    return x ^ (x >> np.uint64(16))


def random_bits(first, n, seed, step, tensor):
    """The 32 random bits of elements first .. first + n - 1 of a tensor at a step."""
    seed = int(seed) & (2 ** 64 - 1)
    word = lambda v: np.uint64(int(v) & 0xFFFFFFFF)  # noqa: E731
    key = word(int(_mixed(word(((seed ^ (seed >> 32)) & 0xFFFFFFFF) + step * 0x9E3779B9))) + tensor * 0xA54FF53B)
    e = np.arange(n, dtype=np.uint64) + np.uint64(first)
    low = ((e & MASK) * np.uint64(0x9E3779B9)) & MASK
    high = ((e >> np.uint64(32)) * np.uint64(0xA54FF53B)) & MASK
    return _mixed((low + high + key) & MASK).astype(np.int64)


def stochastic_e4m3(a, u, never_zero):
    """Magnitudes up to 448 -> e4m3 values: floor(a / width + u) widths, width = distance of the e4m3 values at a."""
    a = np.asarray(a, np.float64)
    width = 2.0 ** (np.maximum(np.frexp(a)[1] - 1, -6) - 3.0)
    k = np.floor(a / width + u)
    if never_zero:
        k = np.where((k == 0) & (a > 0), 1.0, k)
    return np.minimum(k * width, 448.0)


def moment_to_8_bits(a, u, never_zero):
    """fp32 values [n] -> (values of the codes, scales [ceil(n/128)]), scales and products in fp32."""
    a = np.asarray(a, np.float32)
    n = a.size
    pad = np.zeros(-(-n // BLOCK) * BLOCK, np.float32)
    pad[:n] = a
    s, inv = _scale(np.abs(pad.reshape(-1, BLOCK)).max(1))
    scaled = np.minimum(np.abs(pad.reshape(-1, BLOCK) * inv[:, None]).reshape(-1)[:n], TOP)
    return np.copysign(stochastic_e4m3(scaled, u, never_zero), a), s


def adamw(p, g, m, v, lr, step, betas, eps, decay, grad_scale=1.0):
    """fp64 -> new (p, m, v); m, v: the moments' values."""
    b1, b2 = betas
    g = np.asarray(g, np.float64) * grad_scale
    m = b1 * np.asarray(m, np.float64) + (1 - b1) * g
    v = b2 * np.asarray(v, np.float64) + (1 - b2) * g * g
    p = np.asarray(p, np.float64) * (1 - lr * decay) - lr * (m / (1 - b1 ** step)) / (np.sqrt(v / (1 - b2 ** step)) + eps)
    return p, m, v
