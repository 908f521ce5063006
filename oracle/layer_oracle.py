"""CPU oracle of the layer operators (dropout, residual RMS norm, 8-bit blocks and their product).  TEST INFRASTRUCTURE
ONLY, in fp64 (numpy) from the definitions; the HIP library never calls it and shares no code with it.

Pins (tests/test_layer_oracle.py): the published known-answer vectors of Philox4x32-10; the norm's gradient against
differences of the norm; every e4m3 value against its bits and torch's type; hand-worked blocks."""
from __future__ import annotations

import numpy as np


def philox(counter, key):
    """Philox4x32-10 (Salmon, Moraes, Dror, Shaw 2011) on uint64 arrays that hold 32-bit words: four words."""
    low = np.uint64(0xFFFFFFFF)
    x, k = [np.asarray(c, np.uint64) for c in counter], [int(key[0]), int(key[1])]
    for _ in range(10):
        a, b = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(b >> np.uint64(32)) ^ x[1] ^ np.uint64(k[0]), b & low, (a >> np.uint64(32)) ^ x[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) % 2**32, (k[1] + 0xBB67AE85) % 2**32]
    return x


def dropout_threshold(p):
    return int(np.rint(p * 65536.0))


def dropout_keep(rows, d, p, seed, first_row=0):
    """Truth values [rows, d]: the elements that stay."""
    groups = (d + 7) // 8
    row = (np.arange(rows, dtype=np.uint64) + np.uint64(first_row))[:, None] + np.zeros((1, groups), np.uint64)
    col = np.arange(groups, dtype=np.uint64)[None, :] + np.zeros((rows, 1), np.uint64)
    words = philox((col, row & np.uint64(0xFFFFFFFF), row >> np.uint64(32), np.zeros_like(col)), (seed % 2**32, seed >> 32))
    number = np.stack([(w >> np.uint64(s)) & np.uint64(0xFFFF) for w in words for s in (0, 16)], axis=-1)
    return number.reshape(rows, groups * 8)[:, :d] >= dropout_threshold(p)


def dropout(x, p, seed, first_row=0):
    x = np.asarray(x, np.float64)
    t = dropout_threshold(p)
    keep = dropout_keep(x.shape[0], x.shape[1], p, seed, first_row)
    return np.where(keep, x * (65536.0 / (65536 - t)), 0.0)


def rms_norm(h, gain, eps):
    h = np.asarray(h, np.float64)
    return h / np.sqrt((h * h).mean(axis=1, keepdims=True) + eps) * np.asarray(gain, np.float64)


def rms_norm_backward(h, gain, dy, eps):
    """(gradient with respect to h, rows of dy * n, whose sums over a sample's rows are the gain's gradient)."""
    h, gain, dy = (np.asarray(v, np.float64) for v in (h, gain, dy))
    r = 1.0 / np.sqrt((h * h).mean(axis=1, keepdims=True) + eps)
    n = h * r
    w = gain * dy
    return r * (w - n * (w * n).mean(axis=1, keepdims=True)), dy * n


# --------------------------------------------------------------------------------------------------------------------
# 8-bit blocks
# --------------------------------------------------------------------------------------------------------------------

def e4m3_table():
    """The 256 values of e4m3: sign, 4 exponent bits (bias 7), 3 mantissa bits; all ones is NaN, there is no infinity."""
    out = np.empty(256)
    for code in range(256):
        e, m = (code >> 3) & 15, code & 7
        v = np.nan if (code & 127) == 127 else (1 + m / 8) * 2.0 ** (e - 7) if e else m / 8 * 2.0**-6
        out[code] = -v if code > 127 else v
    return out


def block_exponent(big):
    """Biased exponent of a block whose largest finite magnitude is `big`."""
    big = np.asarray(big, np.float64)
    e = np.full(big.shape, -126, np.int64)
    for _ in range(300):
        e += big > 448.0 * np.exp2(e.astype(np.float64))
    return e + 127


def pack(x):
    """x [rows, cols] -> (codes as values [rows, whole blocks], exponents [blocks, rows])."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    blocks = (cols + 127) // 128
    v = np.zeros((rows, blocks * 128))
    v[:, :cols] = x
    v = v.reshape(rows, blocks, 128)
    finite = np.isfinite(v)
    e = block_exponent(np.where(finite, np.abs(v), 0.0).max(axis=2))
    with np.errstate(invalid="ignore"):
        s = v / np.exp2(e - 127.0)[..., None]
        step = np.exp2(np.maximum(np.floor(np.log2(np.maximum(np.abs(np.where(finite, s, 0.0)), 1e-300))), -6.0) - 3.0)
        q = np.where(finite, np.rint(s / step) * step, np.nan)         # rint: ties to even multiples of the step
    return q.reshape(rows, -1), e.T.astype(np.uint8)


def unpack(codes, exponents, cols):
    """uint8 codes [rows, whole blocks] and exponents [blocks, rows] -> what they stand for, [rows, cols]."""
    v = e4m3_table()[codes]
    return (v * np.repeat(np.exp2(exponents.astype(np.float64) - 127.0).T, 128, axis=1))[:, :cols]
