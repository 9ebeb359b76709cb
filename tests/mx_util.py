"""Microscaled 4-bit floating point in 64 bits, written from the format's definition, for the tests."""
import numpy as np

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def blocks(cols):
    return -(-cols // 32)


def pitch(cols):
    return -(-blocks(cols) // 16) * 16


def quantize(x):
    """(codes, scales, values) of a float64 matrix."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    codes = np.zeros((rows, blocks(cols) * 16), dtype=np.uint8)
    scales = np.zeros((rows, pitch(cols)), dtype=np.uint8)
    values = np.zeros((rows, cols))
    for r in range(rows):
        for b in range(blocks(cols)):
            v = x[r, 32 * b:32 * b + 32]
            if not np.isfinite(v).all():
                scales[r, b] = 255
                values[r, 32 * b:32 * b + 32] = np.nan
                continue
            top = np.abs(v).max()
            e = 0 if top == 0 else max(int(np.floor(np.log2(top))) if top >= 2.0 ** -126 else -1000, -125) - 2 + 127
            scales[r, b] = e
            q = np.abs(v) * 2.0 ** (127 - e)
            d = np.abs(q[:, None] - MAGNITUDES[None, :])
            best = d.min(axis=1)
            near = d == best[:, None]
            even = near & (np.arange(8) % 2 == 0)[None, :]
            k = np.where(even.any(axis=1), even.argmax(axis=1), near.argmax(axis=1))       # ties: the even code
            values[r, 32 * b:32 * b + 32] = np.copysign(MAGNITUDES[k] * 2.0 ** (e - 127), v)
            nib = (k + 8 * np.signbit(v)).astype(np.uint8)
            nib = np.pad(nib, (0, 32 - len(nib)))
            codes[r, 16 * b:16 * b + 16] = nib[0::2] | nib[1::2] << 4
    return codes, scales, values


def values_of(codes, scales, cols):
    """The float64 values that codes and scales stand for; a block with scale 255 is NaN."""
    codes = np.asarray(codes)
    nib = np.stack([codes & 15, codes >> 4], axis=2).reshape(codes.shape[0], -1)
    v = MAGNITUDES[nib & 7] * np.where(nib & 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return (v * np.repeat(s[:, :blocks(cols)], 32, axis=1))[:, :cols]


def random_matrix(rows, cols, seed, lo=100, hi=128):
    """Random codes (zero past the last column) and scales 2^(lo-127) .. 2^(hi-127); the bytes past the last block are 255."""
    g = np.random.default_rng(seed)
    nib = g.integers(0, 16, (rows, blocks(cols) * 32), dtype=np.uint8)
    nib[:, cols:] = 0
    scales = np.full((rows, pitch(cols)), 255, dtype=np.uint8)
    scales[:, :blocks(cols)] = g.integers(lo, hi + 1, (rows, blocks(cols)))
    return nib[:, 0::2] | nib[:, 1::2] << 4, scales
