"""fp64 oracle: 4-bit microscaled floating point (OCP MXFP4) and the logits of a
quantised head.

TEST INFRASTRUCTURE ONLY (see the package docstring).

A block of 32 elements has one scale 2^(s - 127) (s a byte, 255 = NaN) and
4-bit codes c = sign, two exponent bits, one mantissa bit:

    value(c) = (-1)^sign * (m / 2                     where the exponent bits are 0
                            (1 + m / 2) 2^(e - 1)     else)

    quantise: s = max(floor(log2 max|x|) - 2, -127) + 127, c the nearest value
              of x / 2^(s - 127), halfway to the even code, beyond 6 to 6
    logits:   z[t, v] = (sum_k h[t, k] w[v, k]) / temperature

Pins (tests/test_policy_oracle.py): the sixteen values listed by hand; every
code and scale quantises to itself; brute force over the sixteen values;
hand-made ties and saturations; the logits against a loop over elements.
"""

from __future__ import annotations

import numpy as np

BLOCK = 32


def mxfp4_code_values() -> np.ndarray:
    """The value of each of the sixteen codes."""
    c = np.arange(16)
    e, m = (c >> 1) & 3, (c & 1).astype(np.float64)
    mag = np.where(e == 0, m / 2, (1 + m / 2) * np.exp2(e - 1.0))
    return np.where(c >> 3 == 1, -mag, mag)


def mxfp4_quantize(x) -> tuple[np.ndarray, np.ndarray]:
    """(codes uint8 [rows, d] one per element, scales uint8 [rows, d / 32]) of rows x."""
    x = np.asarray(x, dtype=np.float64)
    rows, d = x.shape
    b = x.reshape(rows, d // BLOCK, BLOCK)
    bad = ~np.isfinite(b).all(axis=2)
    b = np.where(bad[:, :, None], 0.0, b)
    top = np.abs(b).max(axis=2)
    _, e = np.frexp(top)  # top = m 2^e, 1/2 <= m < 1
    e = np.where(top > 0, np.maximum(e - 1 - 2, -127), -127)
    a = np.abs(b) / np.exp2(e.astype(np.float64))[:, :, None]
    grid = mxfp4_code_values()[:8]
    # the distance to each magnitude; of two equal ones the even code wins
    dist = np.abs(a[..., None] - grid)
    best = dist.min(axis=3, keepdims=True)
    even_first = np.array([0, 2, 4, 6, 1, 3, 5, 7])
    code = even_first[np.argmax((dist == best)[..., even_first], axis=3)]
    code = np.where(np.signbit(b), code + 8, code)
    code = np.where(bad[:, :, None], 0, code)
    scales = np.where(bad, 255, e + 127)
    return code.reshape(rows, d).astype(np.uint8), scales.astype(np.uint8)


def mxfp4_pack(codes) -> np.ndarray:
    """uint8 [rows, d / 2] of one code per element: element 2j in the low half of byte j."""
    return (codes[:, 0::2] | (codes[:, 1::2] << 4)).astype(np.uint8)


def mxfp4_unpack(packed) -> np.ndarray:
    packed = np.asarray(packed)
    out = np.empty((packed.shape[0], packed.shape[1] * 2), dtype=np.uint8)
    out[:, 0::2] = packed & 15
    out[:, 1::2] = packed >> 4
    return out


def mxfp4_values(codes, scales) -> np.ndarray:
    """fp64 values of one code per element [rows, d] and scales [rows, d / 32]."""
    s = np.asarray(scales)
    scale = np.where(s == 255, np.nan, np.exp2(s.astype(np.float64) - 127))
    return mxfp4_code_values()[np.asarray(codes)] * np.repeat(scale, BLOCK, axis=1)


def mxfp4_logits(h, w, temperature: float) -> np.ndarray:
    """fp64 logits of rows h [T, d] and w [V, d] of values."""
    return (np.asarray(h) @ np.asarray(w).T) / float(temperature)
