"""The 4-bit format, the products on it and the norm in 64 bits (numpy), written from the formulas of include/capmoe.h."""
import numpy as np

from fp8_reference import to_bf16  # noqa: F401

BLOCK = 32
MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
E2M1 = np.concatenate([MAGNITUDES, -MAGNITUDES])  # the value of every code


def up(n, m):
    return -(-n // m) * m


def encode(v):
    """64-bit values of magnitude up to 6 to codes: to nearest, ties to the even code; the sign of zero is kept."""
    a = np.abs(v)
    hi = np.clip(np.searchsorted(MAGNITUDES, a), 1, 7)
    lo = hi - 1
    mid = (MAGNITUDES[lo] + MAGNITUDES[hi]) / 2
    code = np.where((a > mid) | ((a == mid) & (hi % 2 == 0)), hi, lo)
    return (code | np.where(np.signbit(v), 8, 0)).astype(np.uint8)


def block_byte(amax):
    """The smallest b >= 0 with amax <= 6 * 2^(b - 127), by trying; 255 for no number."""
    b = np.zeros(amax.shape, np.int64)
    for step in (128, 64, 32, 16, 8, 4, 2, 1):
        worse = amax > 6.0 * np.exp2(b + step - 1 - 127.0)
        b = np.where(worse, b + step, b)
    return np.where(np.isfinite(amax), b, 255)


def scale_places(blocks):
    """Where the byte of each block lies in a row of scales."""
    b = np.arange(blocks)
    return b // 16 * 16 + 4 * (b % 4) + b % 16 // 4


def quantize(x, rows=None):
    """x [.., n, c] -> bytes [.., rows, pitch], scale bytes [.., rows, scale pitch]; rows of zeros behind the n."""
    lead, (n, c) = x.shape[:-2], x.shape[-2:]
    rows = rows or n
    v = np.zeros(lead + (rows, up(c, 256)))
    v[..., :n, :c] = x
    v = v.reshape(v.shape[:-1] + (-1, BLOCK))
    with np.errstate(invalid="ignore"):
        b = block_byte(np.abs(v).max(axis=-1))
    fine = b < 255
    code = encode(np.where(fine[..., None], v, 0) / np.exp2(np.where(fine, b, 127) - 127.0)[..., None])
    code[~fine] = 0
    code = code.reshape(lead + (rows, -1))
    scale = np.zeros(lead + (rows, up(c, 512) // 32), np.uint8)
    scale[..., scale_places(b.shape[-1])] = b
    return code[..., 0::2] | code[..., 1::2] << 4, scale


def quantize_weights(w):
    return quantize(w, up(w.shape[1], 128))


def value(q, scale):
    """The values of 4-bit rows, [.., 2 * pitch]."""
    code = np.stack([q & 15, q >> 4], axis=-1).reshape(q.shape[:-1] + (-1,))
    b = scale[..., scale_places(code.shape[-1] // BLOCK)]
    power = np.where(b == 255, np.nan, np.exp2(b - 127.0))
    return E2M1[code] * np.repeat(power, BLOCK, axis=-1)


def gemm(x, w, offset, token=None):
    """x, w: the values of 4-bit rows and weights.  (y, sum of the magnitudes of the products), rows up to offset[-1]."""
    y, mag = (np.zeros((offset[-1], w.shape[1])) for _ in range(2))
    for e in range(len(offset) - 1):
        rows = np.arange(offset[e], offset[e + 1])
        a = x[rows if token is None else token[rows]]
        y[rows], mag[rows] = a @ w[e].T, np.abs(a) @ np.abs(w[e]).T
    return y, mag


def ffn(x, gate, up_, down, offset, h, token=None):
    """x: the values of 4-bit rows; gate, up_, down: of 4-bit weights; h: the hidden width.  yp up to offset[-1], [*, padded d]."""
    g, u = gemm(x, gate, offset, token)[0], gemm(x, up_, offset, token)[0]
    hidden = to_bf16(g / (1 + np.exp(-g)) * u)[:, :h]
    return gemm(value(*quantize(hidden)), down, offset)[0]


def norm(x, residual, weight, eps, to_type):
    """(h, y before its rounding)"""
    h = x if residual is None else to_type(x + residual)
    y = h / np.sqrt((h ** 2).mean(axis=1, keepdims=True) + eps)
    return h, y if weight is None else y * weight
