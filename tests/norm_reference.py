"""Layer norm and the 8-bit checkpoints in 64 bits on the CPU, from their definitions in include/slope.h."""
import numpy as np

BLOCK = 32


def encode(x):
    """Codes [rows x cols] int8 and exponent bytes [rows x cols/32] of a float64 matrix (values of bf16 or fp32)."""
    rows, cols = x.shape
    blocks = np.asarray(x, np.float64).reshape(rows, cols // BLOCK, BLOCK)
    fine = np.isfinite(blocks).all(-1)
    safe = np.where(fine[..., None], blocks, 0.0)
    largest = np.abs(safe).max(-1)
    # the smallest k in [-126, 121] with largest <= 127.5 * 2^k
    k = np.full(largest.shape, 121, np.int64)
    for candidate in range(120, -127, -1):
        k = np.where(largest <= 127.5 * 2.0 ** candidate, candidate, k)
    codes = np.clip(np.rint(safe / np.ldexp(1.0, k)[..., None]), -127, 127).astype(np.int8)
    return codes.reshape(rows, cols), np.where(fine, k + 127, 255).astype(np.uint8)


def decode(codes, exponents):
    rows, cols = codes.shape
    with np.errstate(invalid="ignore"):
        unit = np.where(exponents == 255, np.nan, np.ldexp(1.0, exponents.astype(np.int64) - 127))
        return (codes.reshape(rows, cols // BLOCK, BLOCK).astype(np.float64) * unit[..., None]).reshape(rows, cols)


def buffer(codes, exponents):
    return np.concatenate([codes.reshape(-1).view(np.uint8), exponents.reshape(-1)])


def split(buf, rows, cols):
    buf = np.asarray(buf, np.uint8)
    return buf[:rows * cols].view(np.int8).reshape(rows, cols), buf[rows * cols:].reshape(rows, cols // BLOCK)


def layer_norm(h, gamma, beta, eps):
    """(y, mean, rstd, xhat) of float64 rows."""
    mean = h.mean(-1)
    rstd = 1.0 / np.sqrt(((h - mean[:, None]) ** 2).mean(-1) + eps)
    xhat = (h - mean[:, None]) * rstd[:, None]
    return xhat * gamma + beta, mean, rstd, xhat


def layer_norm_grads(dy, h, mean, rstd, gamma, dh=None):
    """(dx, dgamma, dbeta, terms): terms bound what rounding in 24 bits is relative to, see the tests."""
    xhat = (h - mean[:, None]) * rstd[:, None]
    g = dy * gamma
    m1, m2 = g.mean(-1, keepdims=True), (g * xhat).mean(-1, keepdims=True)
    dx = rstd[:, None] * (g - m1 - xhat * m2)
    terms = rstd[:, None] * (np.abs(g) + np.abs(g).mean(-1, keepdims=True) + np.abs(xhat) * np.abs(g * xhat).mean(-1, keepdims=True))
    if dh is not None:
        dx, terms = dx + dh, terms + np.abs(dh)
    return dx, (dy * xhat).sum(0), dy.sum(0), terms
