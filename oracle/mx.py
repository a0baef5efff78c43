"""Oracle of the microscaled 4-bit floats, their product, the layer norm and the gradients: numpy, float64, straight from the formulas.
Test infrastructure only.  16-bit inputs come as float64 arrays of their exact values."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BORDER = (GRID[1:] + GRID[:-1]) / 2


def scale_bytes(x):
    """[M, K] -> [M, K/32]: exponent of the largest magnitude less 2, in a byte with bias 127; 255 where the block is not finite."""
    b = np.abs(np.asarray(x, np.float64)).reshape(x.shape[0], -1, 32)
    top = b.max(-1)
    with np.errstate(invalid="ignore"):
        e = np.frexp(np.where(np.isfinite(top), top, 1.0))[1] - 1
    s = np.clip(e - 2 + 127, 0, 254)
    s = np.where(top == 0, 0, s)
    return np.where(np.isfinite(b).all(-1), s, 255).astype(np.uint8)


def encode(x, scales):
    """Codes [M, K] (sign in bit 3) of x under given scale bytes: nearest, ties to the even code, saturating; 0 in blocks of scale 255."""
    s = np.repeat(scales.astype(np.float64), 32, axis=1)
    a = np.where(s == 255, 0.0, np.asarray(x, np.float64))
    q = np.abs(a) * 2.0 ** (127 - s)
    lo, hi = np.searchsorted(BORDER, q, side="left"), np.searchsorted(BORDER, q, side="right")
    code = np.where(lo == hi, lo, np.where(lo % 2 == 0, lo, hi))
    return np.where(s == 255, 0, code + 8 * np.signbit(a)).astype(np.uint8)


def decode(codes, scales):
    s = np.repeat(scales.astype(np.float64), 32, axis=1)
    v = np.where(codes & 8, -1.0, 1.0) * GRID[codes & 7] * 2.0 ** (s - 127)
    return np.where(s == 255, np.nan, v)


def quantize(x):
    s = scale_bytes(x)
    return encode(x, s), s


def values(x):
    return decode(*quantize(x))


def flat(codes):
    """Codes one per byte -> interchange bytes."""
    return (codes[:, 0::2] | codes[:, 1::2] << 4).astype(np.uint8)


def unflat(b):
    return np.stack([b & 15, b >> 4], -1).reshape(b.shape[0], -1)


def linear(a, w, bias=None, residual=None):
    """(Y, sum of the magnitudes that went into each entry) of already quantised values."""
    y, mag = a @ w.T, np.abs(a) @ np.abs(w).T
    for t in (bias, residual):
        if t is not None:
            y, mag = y + t, mag + np.abs(t)
    return y, mag


def linear_grad(dy, w):
    return dy @ w, np.abs(dy) @ np.abs(w)


def norm_stats(x, eps):
    mean = x.mean(-1, keepdims=True)
    d = x - mean
    return mean, 1.0 / np.sqrt((d * d).mean(-1, keepdims=True) + eps)


def norm(x, weight, bias, eps):
    mean, rstd = norm_stats(x, eps)
    return (x - mean) * rstd * weight + bias


def norm_grad(dy, x, weight, mean, rstd, residual=None):
    """(dx, dweight, dbias) with given statistics (columns [M, 1])."""
    xhat = (x - mean) * rstd
    g = dy * weight
    dx = rstd * (g - g.mean(-1, keepdims=True) - xhat * (g * xhat).mean(-1, keepdims=True))
    if residual is not None:
        dx = dx + residual
    return dx, (dy * xhat).sum(0), dy.sum(0)
