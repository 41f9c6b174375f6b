"""fp64 oracle of the operators in front of the loss: layer norm, linear layers, AdamW with moments in 32 or 8 bits.

Plain numpy from the definitions, test infrastructure only (like fcco_oracle)."""
from __future__ import annotations

import math

import numpy as np

BLOCK = 256
M_TOP, V_TOP = 14, 30          # exponent field of a block's largest octave
_erfc = np.frompyfunc(math.erfc, 1, 1)


def layer_norm(x, weight, bias, eps):
    """(y, mean, rstd) of rows x [rows, d]."""
    x = np.asarray(x, np.float64)
    d = x.shape[1]
    mean = x.sum(1) / d
    off = x - mean[:, None]
    rstd = 1.0 / np.sqrt((off * off).sum(1) / d + eps)
    y = off * rstd[:, None]
    if weight is not None:
        y = y * weight
    return (y if bias is None else y + bias), mean, rstd


def layer_norm_grad(x, dy, mean, rstd, weight):
    """(dx, dweight, dbias) with the statistics as given."""
    x, dy = np.asarray(x, np.float64), np.asarray(dy, np.float64)
    xh = (x - np.asarray(mean, np.float64)[:, None]) * np.asarray(rstd, np.float64)[:, None]
    q = dy if weight is None else dy * weight
    dx = q - q.mean(1, keepdims=True) - xh * (q * xh).mean(1, keepdims=True)
    return dx * np.asarray(rstd, np.float64)[:, None], (dy * xh).sum(0), dy.sum(0)


def normal_cdf(z):
    return 0.5 * _erfc(-np.asarray(z, np.float64) / math.sqrt(2.0)).astype(np.float64)


def _gate(z):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-1.702 * z))


def activation(z, act):
    """act: "", "gelu", "quick_gelu"."""
    z = np.asarray(z, np.float64)
    return z * normal_cdf(z) if act == "gelu" else z * _gate(z) if act == "quick_gelu" else z


def activation_slope(z, act):
    z = np.asarray(z, np.float64)
    if act == "gelu":
        return normal_cdf(z) + z * np.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if act == "quick_gelu":
        p = _gate(z)
        return p + 1.702 * z * p * (1.0 - p)
    return np.ones_like(z)


def linear(x, w, bias=None, act="", residual=None):
    """(y, z): z = x w^T + bias, y = act(z) + residual."""
    z = np.asarray(x, np.float64) @ np.asarray(w, np.float64).T
    if bias is not None:
        z = z + bias
    y = activation(z, act)
    return (y if residual is None else y + residual), z


def linear_grad_input(dy, w, pre=None, act=""):
    dx = np.asarray(dy, np.float64) @ np.asarray(w, np.float64)
    return dx * activation_slope(pre, act) if act else dx


def linear_grad_weight(dy, x):
    """(dw, dbias)"""
    dy = np.asarray(dy, np.float64)
    return dy.T @ np.asarray(x, np.float64), dy.sum(0)


# ---- AdamW ---------------------------------------------------------------------------------------------------------

def _grid(top, codes):
    """What the codes 0 .. codes - 1 stand for in a block of exponent 0."""
    return np.array([(c & 7) / 8 * 2.0 ** (1 - top) if c < 8 else (1 + (c & 7) / 8) * 2.0 ** ((c >> 3) - top)
                     for c in range(codes)])


M_GRID, V_GRID = _grid(M_TOP, 128), _grid(V_TOP, 256)


def _spread(exps, n):
    return np.repeat(2.0 ** (np.asarray(exps, np.float64) - 127), BLOCK)[:n]


def decode(codes, exps, second):
    """Values of an 8-bit moment."""
    c = np.asarray(codes).astype(np.int64)
    if second:
        return V_GRID[c] * _spread(exps, c.size)
    return M_GRID[c & 127] * _spread(exps, c.size) * np.where(c >= 128, -1.0, 1.0)


def random_halves(seed, number, n):
    """The 32 random bits of every element of tensor `number`: (low half, high half)."""
    def mix(x):
        x = (x ^ (x >> 16)) * 0x6A09E667 & 0xFFFFFFFF
        x = (x ^ (x >> 15)) * 0xBB67AE85 & 0xFFFFFFFF
        return x ^ (x >> 16)
    key = mix(int(seed + 0x9E3779B9 * (number + 1)) & 0xFFFFFFFF)
    x = np.arange(n, dtype=np.uint64) & 0xFFFFFFFF ^ np.uint64(key)
    x = (x ^ (x >> np.uint64(16))) * np.uint64(0x6A09E667) & np.uint64(0xFFFFFFFF)
    x = (x ^ (x >> np.uint64(15))) * np.uint64(0xBB67AE85) & np.uint64(0xFFFFFFFF)
    x = x ^ (x >> np.uint64(16))
    return (x & np.uint64(0xFFFF)).astype(np.int64), (x >> np.uint64(16)).astype(np.int64)


def encode(x, r16, second):
    """(codes, exponents) of finite values: the grid value below, or the one above where remainder + r / 2^16 >= 1."""
    x = np.asarray(x, np.float64)
    grid = V_GRID if second else M_GRID
    codes, exps = np.zeros(x.size, np.uint8), []
    for at in range(0, x.size, BLOCK):
        part = x[at:at + BLOCK]
        size = np.abs(part)
        top = size.max()
        k = min(126, max(-94, math.frexp(top)[1] - 1 if top > 0 else -94))
        y = size * 2.0 ** -k
        below = np.minimum(np.searchsorted(grid, y, side="right") - 1, grid.size - 2)
        share = (y - grid[below]) / (grid[below + 1] - grid[below])
        c = below + (share + r16[at:at + BLOCK] / 65536.0 >= 1.0)
        c = np.minimum(c, grid.size - 1)
        if second:
            c = np.where((part > 0) & (c == 0), 1, c)
        else:
            c = c + 128 * (part < 0)
        codes[at:at + BLOCK] = c
        exps.append(k + 127)
    return codes, np.array(exps, np.uint8)


def adamw(p, g, m, v, *, step, lr, beta1, beta2, eps, weight_decay):
    """(p, m, v) after a step, everything in fp64; scalars as the fp32 numbers that a configuration holds."""
    lr, beta1, beta2, eps, wd = (float(np.float32(s)) for s in (lr, beta1, beta2, eps, weight_decay))
    p, g, m, v = (np.asarray(t, np.float64) for t in (p, g, m, v))
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    p = p - lr * wd * p - lr * (m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps)
    return p, m, v
