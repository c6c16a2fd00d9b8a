"""Microscaled operands and the norm in front of them, from their definitions, in 64 bits (numpy).

TEST INFRASTRUCTURE ONLY, like quest_oracle.py.  A group of 32 consecutive elements shares the scale 2^e,
e = floor(log2(largest magnitude)) - (exponent of the format's largest element), at least -127; codes are the nearest
elements (ties to the even code, clipped); an element is trusted up to the largest element and half the interval below it.
"""
from __future__ import annotations

import numpy as np

GROUP = 32
E2M1, E4M3 = 0, 1


def _magnitudes(fmt: int) -> np.ndarray:
    """Magnitudes of the codes 0, 1, .. without their sign, ascending."""
    exponent_bits, mantissa_bits, bias = (2, 1, 1) if fmt == E2M1 else (4, 3, 7)
    values = []
    for e in range(1 << exponent_bits):
        for m in range(1 << mantissa_bits):
            fraction = m / (1 << mantissa_bits)
            values.append(fraction * 2.0 ** (1 - bias) if e == 0 else (1 + fraction) * 2.0 ** (e - bias))
    return np.array(values[:-1] if fmt == E4M3 else values)      # E4M3: the highest code is NaN


MAGNITUDES = (_magnitudes(E2M1), _magnitudes(E4M3))
LARGEST_EXPONENT = (2, 8)
TRUSTED = tuple(m[-1] + (m[-1] - m[-2]) / 2 for m in MAGNITUDES)


def _nearest_code(a: np.ndarray, fmt: int) -> np.ndarray:
    grid = MAGNITUDES[fmt]
    mid = (grid[1:] + grid[:-1]) / 2
    code = np.searchsorted(mid, a, side="left")                  # a tie goes to the lower code ..
    tie = (code < len(mid)) & (a == mid[np.minimum(code, len(mid) - 1)])
    return np.where(tie & (code % 2 == 1), code + 1, code)       # .. unless that is odd


def quantize(xh: np.ndarray, fmt: int):
    """(codes without packing, scale bytes, trust) of rows in 64 bits (or in fp32: their values are taken as they are)."""
    xh = np.asarray(xh, dtype=np.float64)
    rows, cols = xh.shape
    g = xh.reshape(rows, cols // GROUP, GROUP)
    finite = np.isfinite(g).all(-1, keepdims=True)
    g = np.where(finite, g, 0.0)
    largest = np.abs(g).max(-1, keepdims=True)
    _, exponent = np.frexp(largest)
    exponent = np.where(largest == 0, -127, np.maximum(exponent - 1 - LARGEST_EXPONENT[fmt], -127))
    t = np.ldexp(g, -exponent)
    code = _nearest_code(np.abs(t), fmt) | (np.signbit(t).astype(np.int64) << (3 if fmt == E2M1 else 7))
    trust = (np.abs(t) <= TRUSTED[fmt]) & finite
    scales = np.where(finite, exponent + 127, 255)[..., 0].astype(np.uint8)
    code = np.where(finite, code, 0)
    return code.reshape(rows, cols).astype(np.uint8), scales, trust.reshape(rows, cols)


def pack(code: np.ndarray, fmt: int) -> np.ndarray:
    return code.astype(np.uint8) if fmt == E4M3 else (code[:, 0::2] | (code[:, 1::2] << 4)).astype(np.uint8)


def unpack(codes: np.ndarray, fmt: int) -> np.ndarray:
    if fmt == E4M3:
        return codes
    return np.stack([codes & 15, codes >> 4], axis=-1).reshape(codes.shape[0], -1)


def values(codes: np.ndarray, scales: np.ndarray, fmt: int) -> np.ndarray:
    """What packed codes and scale bytes stand for."""
    code = unpack(codes, fmt)
    sign_bit = 8 if fmt == E2M1 else 128
    grid = np.append(MAGNITUDES[fmt], np.nan) if fmt == E4M3 else MAGNITUDES[fmt]
    v = np.where(code & sign_bit, -1.0, 1.0) * grid[code & (sign_bit - 1)]
    scale = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return v * np.repeat(scale, GROUP, axis=1)


def pack_mask(trust: np.ndarray) -> np.ndarray:
    return np.packbits(trust, axis=1, bitorder="little")


def hadamard_f32(x: np.ndarray, n: int) -> np.ndarray:
    """The block transform in fp32, strides 1, 2, .. n / 2 and then the factor: its rounding is part of the definition of which
    side of a border a value falls."""
    x = np.asarray(x, dtype=np.float32)
    rows, cols = x.shape
    h = 1
    while h < n:
        v = x.reshape(rows, cols // (2 * h), 2, h)
        x = np.stack([v[:, :, 0] + v[:, :, 1], v[:, :, 0] - v[:, :, 1]], axis=2).reshape(rows, cols)
        h *= 2
    return x if n == 1 else x * np.float32(1.0 / np.sqrt(float(n)))


def rms_norm(h: np.ndarray, weight: np.ndarray, eps: float):
    """(y, rstd) in 64 bits."""
    mean = (h * h).mean(-1) + eps
    with np.errstate(divide="ignore"):
        rstd = np.where(mean == 0, 0.0, 1.0 / np.sqrt(mean))
    return h * rstd[:, None] * weight, rstd


def rms_norm_backward(dy: np.ndarray, h: np.ndarray, weight: np.ndarray, rstd: np.ndarray, dh: np.ndarray | None = None):
    """(dx, dweight) in 64 bits."""
    xhat = h * rstd[:, None]
    t = dy * weight
    dx = rstd[:, None] * (t - xhat * (t * xhat).mean(-1, keepdims=True))
    return dx if dh is None else dx + dh, (dy * xhat).sum(0)
