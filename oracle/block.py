"""Oracle of what stands around the microscaled linears of a transformer block: head norms with rotation, activations and gates, products by expert, and their
gradients: numpy, float64, straight from the formulas.  Test infrastructure only.  16-bit inputs come as float64 arrays of their exact values."""
import math

import numpy as np

from . import mx


def frequencies(sections, theta=10000.0, restart=True):
    """Radians of every pair for one position, and the axis that it goes by."""
    total = sum(sections)
    f = [theta ** (-i / n) for n in sections for i in range(n)] if restart else [theta ** (-i / total) for i in range(total)]
    return np.array(f), np.repeat(np.arange(len(sections)), sections)


def angles(positions, freq, axis):
    """[M, pairs], modulo a turn in the products of whole numbers and doubles: math.fmod keeps far positions exact to 2^-53 of the product."""
    a = positions.astype(np.float64)[:, axis] * freq
    return np.fmod(a, 2 * math.pi)


def pairs(D, P, interleaved):
    """Columns of the first and the second value of every pair."""
    i = np.arange(P)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + P)


def turn(u, angle, interleaved):
    """u [M, heads, D], angle [M, P]."""
    a, b = pairs(u.shape[-1], angle.shape[1], interleaved)
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    o = u.copy()
    o[..., a], o[..., b] = u[..., a] * c - u[..., b] * s, u[..., a] * s + u[..., b] * c
    return o


def heads(x, w, angle, interleaved, eps, norm=True):
    """x [M, heads, D], w [heads, D]."""
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps) if norm else np.ones(x.shape[:2] + (1,))
    return turn(x * r * w, angle, interleaved)


def heads_grad(dy, x, w, angle, interleaved, eps, norm=True):
    """(dx, dw [heads, D])"""
    g = turn(dy, -angle, interleaved)
    if not norm:
        return g, None
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return r * (g * w - x * r * r * (g * w * x).mean(-1, keepdims=True)), (g * x * r).sum(0)


_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def tail(a):
    """Phi(-|a|)"""
    return 0.5 * _erfc(np.abs(a) / math.sqrt(2.0))


def gauss(a):
    return np.exp(-0.5 * a * a) / math.sqrt(2.0 * math.pi)


def logistic_terms(act):
    """silu and gelu_tanh are a s(c a + d a^3), s the logistic function: tanh(z) = 2 s(2 z) - 1."""
    k = 2.0 * math.sqrt(2.0 / math.pi)
    return (1.0, 0.0) if act == "silu" else (k, k * 0.044715)


def logistic(z):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-z))


def act(a, name):
    if name is None:
        return a
    if name == "gelu":
        return a * np.where(a < 0, tail(a), 1.0 - tail(a))
    c, d = logistic_terms(name)
    return a * logistic(c * a + d * a ** 3)


def slope(a, name):
    if name == "gelu":
        return np.where(a < 0, tail(a), 1.0 - tail(a)) + a * gauss(a)
    c, d = logistic_terms(name)
    s, other = logistic(c * a + d * a ** 3), logistic(-(c * a + d * a ** 3))
    return s + a * s * other * (c + 3 * d * a * a)


def halves(a):
    return a[:, :a.shape[1] // 2], a[:, a.shape[1] // 2:]


def activated(a, name, gated):
    if not gated:
        return act(a, name)
    v, g = halves(a)
    return v * act(g, name)


def act_grad(dy, a, name, gated):
    if not gated:
        return dy * slope(a, name)
    v, g = halves(a)
    return np.concatenate((dy * act(g, name), dy * v * slope(g, name)), 1)


def grouped(a, w, offsets, bias=None):
    """Quantised values a [M, K] and w [experts, N, K]: (sums, magnitudes) [M, N], NaN and 0 in rows that no expert has."""
    M, N = a.shape[0], w.shape[1]
    y, mag = np.full((M, N), np.nan), np.zeros((M, N))
    for e in range(w.shape[0]):
        r = slice(offsets[e], offsets[e + 1])
        y[r], mag[r] = mx.linear(a[r], w[e], None if bias is None else bias[e])
    return y, mag


def grouped_grad(dy, w, offsets):
    M, K = dy.shape[0], w.shape[2]
    dx, mag = np.full((M, K), np.nan), np.zeros((M, K))
    for e in range(w.shape[0]):
        r = slice(offsets[e], offsets[e + 1])
        dx[r], mag[r] = mx.linear_grad(dy[r], w[e])
    return dx, mag
