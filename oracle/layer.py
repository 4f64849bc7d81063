"""The operators of a transformer layer around the attention, in fp64 from their definitions: root-mean-square norm, matrix
product with its epilogue, rotary positions with several axes, and their gradients.  Test infrastructure; shares nothing with the library."""
import math

import numpy as np


def oracle_axes(sections, order):
    """The axis of every pair."""
    if order == "blocks":
        return np.repeat(np.arange(len(sections)), sections)
    axis = []
    for i in range(sum(sections)):
        a = i % len(sections)
        axis.append(a if i < len(sections) * sections[a] else 0)
    return np.array(axis, dtype=np.int64)


def oracle_rope_axes(x, positions, axis, freq, scale, layout="half", inverse=False):
    """x [rows, heads, d], positions [axes, rows] -> fp64."""
    y = np.array(x, dtype=np.float64)
    n = len(freq)
    i = np.arange(n)
    a, b = (i, i + n) if layout == "half" else (2 * i, 2 * i + 1)
    at = np.asarray(positions, dtype=np.float64)[axis].T            # [rows, pairs]
    turn = scale * np.exp((-1j if inverse else 1j) * at * freq)[:, None, :]
    z = (y[..., a] + 1j * y[..., b]) * turn
    y[..., a], y[..., b] = z.real, z.imag
    return y


def oracle_rms(h, weight, eps):
    """(y, 1 / root mean square) of the last axis."""
    h = np.asarray(h, dtype=np.float64)
    r = 1.0 / np.sqrt((h * h).mean(-1, keepdims=True) + eps)
    return h * r * weight, r


def oracle_rms_bwd(h, weight, d_y, eps, d_summed=0.0):
    """(d_h, d_weight): d_h[j] = sum_i dy[i] w[i] d(h[i] r)/d h[j] + d_summed[j], d r / d h[j] = -r^3 h[j] / n."""
    h, d_y = np.asarray(h, dtype=np.float64), np.asarray(d_y, dtype=np.float64)
    n = h.shape[-1]
    r = 1.0 / np.sqrt((h * h).mean(-1, keepdims=True) + eps)
    g = d_y * weight
    d_h = g * r - r ** 3 * h * (g * h).sum(-1, keepdims=True) / n + d_summed
    return d_h, (d_y * h * r).reshape(-1, n).sum(0)


def _sigmoid(z):
    e = np.exp(-np.abs(z))
    return np.where(z >= 0, 1.0 / (1.0 + e), e / (1.0 + e))


_erf = np.vectorize(math.erf, otypes=[np.float64])


def oracle_act(z, activation):
    """(value, slope)"""
    z = np.asarray(z, dtype=np.float64)
    if activation is None:
        return z, np.ones_like(z)
    if activation == "relu":
        return np.maximum(z, 0.0), (z > 0).astype(np.float64)
    if activation == "silu":
        s = _sigmoid(z)
        return z * s, s + z * s * (1.0 - s)
    if activation == "gelu":
        c = 0.5 * (1.0 + _erf(z / math.sqrt(2.0)))
        return z * c, c + z * np.exp(-z * z / 2.0) / math.sqrt(2.0 * math.pi)
    k = math.sqrt(2.0 / math.pi)
    t = np.tanh(k * (z + 0.044715 * z ** 3))
    return 0.5 * z * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * k * (1.0 + 3.0 * 0.044715 * z * z)


def oracle_linear(x, weight, bias=None, activation=None, mul=None, residual=None):
    """(y, z)"""
    z = np.asarray(x, dtype=np.float64) @ np.asarray(weight, dtype=np.float64).T
    if bias is not None:
        z = z + bias
    y = oracle_act(z, activation)[0]
    if mul is not None:
        y = y * mul
    if residual is not None:
        y = y + residual
    return y, z


def oracle_linear_bwd(x, weight, d_y, z=None, activation=None, mul=None):
    """(d_x, d_weight, d_bias, d_mul) at the given z"""
    d_y = np.asarray(d_y, dtype=np.float64)
    dz, d_mul = d_y, None
    if activation is not None or mul is not None:
        value, slope = oracle_act(z, activation)
        if mul is not None:
            d_mul, dz = d_y * value, dz * mul
        dz = dz * slope
    return dz @ weight, dz.T @ np.asarray(x, dtype=np.float64), dz.sum(0), d_mul
