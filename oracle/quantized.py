"""Rows of 4-bit floats with a scale for every 32 dimensions, in 64 bits: TEST INFRASTRUCTURE ONLY (see the package).

Written from the definitions in ``include/hdc.h``, element by element: an element is compared with the eight
magnitudes, a code is looked up, a product is a sum over the dimensions."""
from __future__ import annotations

import numpy as np

MAGNITUDES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def quantize(rows):
    """(codes u32 [N][4 W], scales u8 [N][W], values f64 [N][D], norms f64 [N]) of fp32 rows [N][D]."""
    rows = np.asarray(rows, np.float32)
    N, D = rows.shape
    W = (D + 31) // 32
    x = np.zeros((N, 32 * W), np.float32)
    x[:, :D] = rows
    x = x.reshape(N, W, 32)
    fine = np.isfinite(x).all(2)
    safe = np.where(fine[:, :, None], x, 0).astype(np.float64)
    most = np.abs(safe).max(2)
    e = np.maximum(np.where(most > 0, np.frexp(most)[1] - 1, -1000) - 2, -127)
    v = np.abs(safe) / np.exp2(e.astype(np.float64))[:, :, None]
    far = np.abs(np.minimum(v, 6.0)[..., None] - MAGNITUDES)                  # of every magnitude
    near = far == far.min(-1, keepdims=True)                                    # one of them, or two neighbours
    low = near.argmax(-1)
    code = np.where((near.sum(-1) == 2) & (low % 2 == 1), low + 1, low)         # halfway: the even one
    code = np.where(fine[:, :, None], code + 8 * np.signbit(safe), 0)
    scales = np.where(fine, e + 127, 255).astype(np.uint8)
    codes = np.zeros((N, W, 4), np.uint64)
    for i in range(32):
        codes[:, :, i % 4] |= code[:, :, i].astype(np.uint64) << np.uint64(4 * (i // 4))
    codes = codes.astype(np.uint32).reshape(N, 4 * W)
    v = values(codes, scales, D)
    return codes, scales, v, (v * v).sum(1)


def values(codes, scales, D):
    """What codes and scales stand for, f64 [N][D]; a block of scale 255 is no numbers."""
    codes = np.asarray(codes).view(np.uint32)
    N, W = scales.shape
    words = codes.reshape(N, W, 4)
    v = np.empty((N, W, 32))
    for i in range(32):
        code = words[:, :, i % 4] >> np.uint32(4 * (i // 4)) & np.uint32(15)
        v[:, :, i] = np.where(code & 8, -MAGNITUDES[code & 7], MAGNITUDES[code & 7])
    unit = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    with np.errstate(invalid="ignore"):
        return (v * unit[:, :, None]).reshape(N, 32 * W)[:, :D]


def signs(hv, D):
    return 2.0 * np.unpackbits(np.ascontiguousarray(hv).view(np.uint8), axis=1, bitorder="little")[:, :D] - 1.0


def cosines(hv, v, norm):
    """cos f64 [N][C] of hypervectors with rows v [C][D]; 0 for a row of zeros."""
    with np.errstate(invalid="ignore", divide="ignore"):
        return np.where(norm == 0, 0.0, signs(hv, v.shape[1]) @ v.T / (np.sqrt(norm) * np.sqrt(v.shape[1])))


def nearest(cos):
    return np.where(np.isnan(cos), -np.inf, cos).argmax(1).astype(np.int32)


def train_batch(hv, labels, acc, lr):
    """(fp32 rows after one batch, the sum of the magnitudes of the weights that each row took)."""
    C, D = acc.shape
    _, _, v, norm = quantize(acc)
    cos = cosines(hv, v, norm)
    pred = nearest(cos)
    weight = np.zeros((len(labels), C))
    for n, (y, p) in enumerate(zip(labels, pred)):
        if 0 <= y < C:
            weight[n, y] = np.float32(1.0 - cos[n, y])
            if p != y:
                weight[n, p] = -np.float64(np.float32(np.float64(np.float32(lr)) * (1.0 - cos[n, p])))
    return (acc.astype(np.float64) + weight.T @ signs(hv, D)).astype(np.float32), np.abs(weight).sum(0)
