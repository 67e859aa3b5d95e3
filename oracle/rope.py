"""Oracle: rotary positions in float64 (no library code).

Of each head the first r dims turn: pair i = 0 .. r/2 - 1 by p f_i radians at position p, as the complex
number a + i b times amplitude e^(i p f_i). A pair is dims (i, i + r/2), or (2 i, 2 i + 1). The frequencies
are base^(-2 i / r), for longer contexts divided by a factor (linear), of a larger base (ntk), or divided
only where a pair makes few turns over the original context (parts).
"""
from __future__ import annotations

import math

import numpy as np


def frequencies(r: int, base: float, scaling: str = "none", factor: float = 1.0, original_len: float = 0.0,
                low: float = 1.0, high: float = 32.0):
    """(frequencies [r/2], amplitude)"""
    if scaling == "ntk":
        base = base * factor ** (r / (r - 2))
    f = np.array([base ** (-2 * i / r) for i in range(r // 2)])
    if scaling == "linear":
        return f / factor, 1.0
    if scaling == "parts":
        out = []
        for x in f:
            turns = original_len / (2 * math.pi / x)
            keep = 0.0 if turns < low else 1.0 if turns > high else (turns - low) / (high - low)
            out.append(keep * x + (1 - keep) * x / factor)
        return np.array(out), 1 + 0.1 * math.log(factor)
    return f, 1.0


def rotate(x: np.ndarray, pos, f: np.ndarray, amplitude: float = 1.0, interleaved: bool = False) -> np.ndarray:
    """x [..., rows, heads, d] at positions pos [rows]."""
    x = np.array(x, dtype=np.float64)
    r = 2 * len(f)
    first, second = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    angle = np.asarray(pos, dtype=np.float64)[:, None, None] * f
    z = (x[..., first] + 1j * x[..., second]) * (amplitude * np.exp(1j * angle))
    x[..., first], x[..., second] = z.real, z.imag
    return x
