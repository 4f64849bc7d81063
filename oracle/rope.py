"""Rotary positions in fp64, from the definition: pair i of a row at position p is the complex number x1 + i x2 times
scale * exp(i p f_i).  Test infrastructure; shares nothing with the library."""
import math

import numpy as np


def oracle_rope_frequencies(rotary_dim, base, scaling=None, factor=1.0, original_positions=0, low=0.0, high=0.0,
                            attention_scale=0.0):
    """(radians per position of every pair, factor on cos and sin)."""
    n = rotary_dim // 2
    scale = 1.0
    if scaling == "ntk":
        base = base * factor ** (rotary_dim / (rotary_dim - 2.0))
    freq = [1.0 / base ** (2.0 * i / rotary_dim) for i in range(n)]
    if scaling == "linear":
        freq = [f / factor for f in freq]
    if scaling in ("yarn", "banded"):
        low = low or 1.0
        high = high or (32.0 if scaling == "yarn" else 4.0)
        # the pair index at which a pair makes `turns` turns over the original length
        index = lambda turns: rotary_dim * math.log(original_positions / (2 * math.pi * turns)) / (2 * math.log(base))
        first, last = max(math.floor(index(high)), 0), min(math.ceil(index(low)), rotary_dim - 1)
        for i in range(n):
            if scaling == "yarn":
                stretch = (i - first) / max(last - first, 0.001)
            else:
                stretch = (high - original_positions * freq[i] / (2 * math.pi)) / (high - low)
            stretch = min(max(stretch, 0.0), 1.0)
            freq[i] = (1 - stretch) * freq[i] + stretch * freq[i] / factor
        if scaling == "yarn":
            scale = 1.0 + 0.1 * math.log(factor)
    return np.array(freq), attention_scale or scale


def oracle_rope(x, positions, freq, scale, layout="half", inverse=False):
    """x [rows, heads, d] (any float type) -> fp64."""
    y = np.array(x, dtype=np.float64)
    n = len(freq)
    i = np.arange(n)
    a, b = (i, i + n) if layout == "half" else (2 * i, 2 * i + 1)
    angle = np.multiply.outer(np.asarray(positions, dtype=np.float64), freq)[:, None, :]
    turn = scale * np.exp((-1j if inverse else 1j) * angle)
    z = (y[..., a] + 1j * y[..., b]) * turn
    y[..., a], y[..., b] = z.real, z.imag
    return y
