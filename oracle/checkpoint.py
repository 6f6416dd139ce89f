"""Activations in e4m3 with one power of two for every 32 consecutive features of a row, from the definition.

Test infrastructure only (see the package header).

    e = the least exponent >= -117 with max |x| <= 448 * 2^e over the block's finite elements
    code = RNE_e4m3(x * 2^-e), scale byte = e + 127; infinities and NaN become NaN codes
"""
import numpy as np

from . import formats as F

BLOCK = 32
LEAST = -117


def pack(x):
    """float64 (R, C) -> (codes uint8 (R, C), scales uint8 (R, ceil(C / 32)))."""
    R, C = x.shape
    codes, scales = np.zeros((R, C), dtype=np.uint8), np.zeros((R, -(-C // BLOCK)), dtype=np.uint8)
    for b in range(scales.shape[1]):
        v = x[:, b * BLOCK:(b + 1) * BLOCK]
        fine = np.isfinite(v)
        top = np.max(np.abs(np.where(fine, v, 0.0)), axis=1, initial=0.0)
        e = np.full(R, LEAST)
        while True:                                                    # the definition, one exponent at a time
            more = top > 448.0 * np.exp2(e.astype(np.float64))
            if not more.any():
                break
            e = np.where(more, e + 1, e)
        q = np.where(fine, v, 0.0) * np.exp2(-e.astype(np.float64))[:, None]
        codes[:, b * BLOCK:(b + 1) * BLOCK] = np.where(fine, F.f32_to_e4m3_rne_sat(q.astype(np.float32)), 0x7F)
        scales[:, b] = e + 127
    return codes, scales


def decode(codes, scales):
    """float64 values of the codes."""
    step = np.exp2(scales.astype(np.float64) - 127.0)
    return F.e4m3_to_f32(codes).astype(np.float64) * np.repeat(step, BLOCK, axis=1)[:, :codes.shape[1]]
