"""The 8-bit format and the products on it in 64 bits (numpy), written from the formulas of include/capmoe.h."""
import numpy as np

BLOCK = 128
# the value of every byte
_b = np.arange(256)
_e, _m, _s = (_b >> 3) & 15, _b & 7, np.where(_b & 128, -1.0, 1.0)
E4M3 = _s * np.where(_e > 0, (1 + _m / 8.0) * 2.0 ** (_e - 7.0), _m / 8.0 * 2.0 ** -6)
E4M3[(_b & 127) == 127] = np.nan


def up(n, m=BLOCK):
    return -(-n // m) * m


def scale_pitch(cols):
    return 4 * -(-cols // 512)


def encode(v):
    """64-bit values of magnitude up to 448 (or NaN) to bytes: to nearest, ties to the even byte; the sign of zero is kept."""
    mags = E4M3[:127]
    a = np.abs(v)
    hi = np.clip(np.searchsorted(mags, np.where(np.isnan(a), 0, a)), 1, 126)
    lo = hi - 1
    mid = (mags[lo] + mags[hi]) / 2
    byte = np.where((a > mid) | ((a == mid) & (hi % 2 == 0)), hi, lo)
    byte = np.where(np.isnan(v), 127, byte | np.where(np.signbit(v), 128, 0))
    return byte.astype(np.uint8)


def block_byte(amax):
    """The smallest b >= 0 with amax <= 448 * 2^(b - 127), by trying."""
    b = np.zeros(amax.shape, np.int64)
    for step in (128, 64, 32, 16, 8, 4, 2, 1):
        worse = amax > 448.0 * np.exp2(b + step - 1 - 127.0)
        b = np.where(worse, b + step, b)
    return b


def quantize_blocks(v, axes):
    """(bytes of the values, scale bytes with the axes kept) of blocks that lie along `axes`."""
    fine = np.isfinite(v)
    b = block_byte(np.abs(np.where(fine, v, 0.0)).max(axis=axes, keepdims=True))
    q = encode(np.where(fine, v / np.exp2(b - 127.0), np.nan))
    return q, b


def quantize_rows(x):
    r, c = x.shape
    v = np.zeros((r, up(c)))
    v[:, :c] = x
    q, b = quantize_blocks(v.reshape(r, -1, BLOCK), (2,))
    s = np.zeros((r, scale_pitch(c)), np.uint8)
    s[:, : b.shape[1]] = b[:, :, 0]
    return q.reshape(r, -1), s


def quantize_weights(w):
    e, n, k = w.shape
    v = np.zeros((e, up(n), up(k)))
    v[:, :n, :k] = w
    q, b = quantize_blocks(v.reshape(e, up(n) // BLOCK, BLOCK, up(k) // BLOCK, BLOCK), (2, 4))
    s = np.zeros((e, up(n) // BLOCK, scale_pitch(k)), np.uint8)
    s[:, :, : up(k) // BLOCK] = b[:, :, 0, :, 0]
    return q.reshape(v.shape), s


def rows_value(q, s):
    kb = q.shape[1] // BLOCK
    return E4M3[q] * np.repeat(np.exp2(s[:, :kb] - 127.0), BLOCK, axis=1)


def weights_value(q, s):
    kb = q.shape[2] // BLOCK
    return E4M3[q] * np.repeat(np.repeat(np.exp2(s[:, :, :kb] - 127.0), BLOCK, axis=1), BLOCK, axis=2)


def to_bf16(v):
    """64-bit values rounded once to bf16 (normal range)."""
    m, e = np.frexp(v)
    return np.ldexp(np.rint(m * 256), e - 8)


def gemm(x, w, offset, token=None):
    """x, w: the values of 8-bit rows and weights.  (y, sum of the magnitudes of the products), rows up to offset[-1]."""
    y, mag = (np.zeros((offset[-1], w.shape[1])) for _ in range(2))
    for e in range(len(offset) - 1):
        rows = np.arange(offset[e], offset[e + 1])
        a = x[rows if token is None else token[rows]]
        y[rows], mag[rows] = a @ w[e].T, np.abs(a) @ np.abs(w[e]).T
    return y, mag


def ffn(x, gate, up_, down, offset, token=None):
    """x [*, d] as it is; gate, up_, down: the values of 8-bit weights.  yp up to offset[-1], [*, padded d]."""
    xv = rows_value(*quantize_rows(x))
    g, u = gemm(xv, gate, offset, token)[0], gemm(xv, up_, offset, token)[0]
    hidden = rows_value(*quantize_rows(to_bf16(g / (1 + np.exp(-g)) * u)))
    return gemm(hidden, down, offset)[0]
