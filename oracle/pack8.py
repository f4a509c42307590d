"""8-bit checkpoints in fp64: test infrastructure."""
from __future__ import annotations

import math

import numpy as np


def pack(x):
    """(codes, scale bytes) of x [rows, cols]: blocks of 32, the smallest power of two 2^e with 127 2^e >= max |x|."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    blocks = -(-cols // 32)
    codes, scales = np.zeros((rows, cols), np.int8), np.zeros((rows, blocks), np.uint8)
    for i in range(rows):
        for j in range(blocks):
            v = x[i, 32 * j:32 * j + 32]
            if not np.isfinite(v).all():
                scales[i, j] = 255
                continue
            big, e = np.abs(v).max(), -126
            if big > 0:
                e = max(e, math.frexp(big)[1] - 9)
                while e < 121 and 127.0 * 2.0 ** e < big:
                    e += 1
            scales[i, j] = e + 127
            codes[i, 32 * j:32 * j + 32] = np.clip(np.rint(v / 2.0 ** e), -127, 127)
    return codes, scales


def unpack(codes, scales):
    unit = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127)).repeat(32, 1)[:, :codes.shape[1]]
    return codes * unit


def through(x):
    """What x [.., n] is after being packed and read back."""
    x = np.asarray(x, np.float64)
    return unpack(*pack(x.reshape(-1, x.shape[-1]))).reshape(x.shape)
