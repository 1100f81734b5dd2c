"""Restatement of the position rotation and of the 4-bit form of cached rows, in
plain numpy, written from the definitions; shares no code with the CUDA path."""

from __future__ import annotations

import numpy as np

GROUP = 32
F = np.float32


def rotate(x, angles_cos, angles_sin, interleaved, dtype):
    """x [..., D]; the cosines and sines [..., pairs] of its pairs.  Every
    operation in ``dtype``; the dimensions behind the pairs stay as they are."""
    x = np.asarray(x, dtype)
    c, s = np.asarray(angles_cos, dtype), np.asarray(angles_sin, dtype)
    pairs = c.shape[-1]
    y = x.copy()
    a_at = slice(0, 2 * pairs, 2) if interleaved else slice(0, pairs)
    b_at = slice(1, 2 * pairs, 2) if interleaved else slice(pairs, 2 * pairs)
    a, b = x[..., a_at], x[..., b_at]
    y[..., a_at] = a * c - b * s
    y[..., b_at] = b * c + a * s
    return y


def four_bits_up(t):
    """The least float32 of four significant bits that is not below t >= 0."""
    t = np.asarray(t, F)
    m, e = np.frexp(t.astype(np.float64))     # t = m 2^e, m in [1/2, 1)
    return np.ldexp(np.ceil(m * 16) / 16, e).astype(F)


def quantise(x):
    """x [..., D] float32 -> (codes 0..15 [..., D], scales float32 [..., D/32])."""
    g = np.asarray(x, F).reshape(*x.shape[:-1], x.shape[-1] // GROUP, GROUP)
    nan = np.isnan(g).any(-1)
    top = np.abs(np.where(np.isnan(g), 0, g)).max(-1).astype(F)
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        t = top * F(1 / 7.5)
        step = np.where(np.isinf(t), F(61440), four_bits_up(np.where(np.isinf(t), 0, t)))
        step = np.minimum(np.maximum(step, F(2.0 ** -14)), F(61440)).astype(F)
        code = np.rint(g * (F(1) / step)[..., None])
    code = np.clip(np.where(np.isnan(code), 0, code), -8, 7).astype(np.int64) + 8
    return code.reshape(x.shape), np.where(nan, F("nan"), step)


def values(codes, scales):
    """What the codes and scales hold, in float64."""
    g = codes.reshape(*codes.shape[:-1], codes.shape[-1] // GROUP, GROUP).astype(np.float64) - 8.0
    return (g * np.asarray(scales, np.float64)[..., None]).reshape(codes.shape)


def pack(codes):
    """Codes [..., D] as bytes [..., D/2], even dimensions in the low half."""
    return (codes[..., 0::2] | (codes[..., 1::2] << 4)).astype(np.uint8)


def unpack(byts):
    b = np.asarray(byts).astype(np.int64)
    return np.stack([b & 15, b >> 4], -1).reshape(*b.shape[:-1], 2 * b.shape[-1])
