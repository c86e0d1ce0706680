"""The layer operators in 64 bits on the CPU (test infrastructure only): numpy, from the formulas.

Packed matrices have the layout of include/pp_layer.h.  Nothing here is shared with the library.
"""
import math

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
GRID = np.array([-6.0, -4.0, -3.0, -2.0, -1.5, -1.0, -0.5, 0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def nearest_e2m1(a):
    """Index of the nearest entry of E2M1 to a >= 0, ties to the even index, the last beyond the last."""
    d = np.abs(a[..., None] - E2M1)
    low = d.min(-1, keepdims=True)
    tied = d == low                                   # exact: a and the entries are short binary fractions
    even = tied & (np.arange(8) % 2 == 0)
    return np.where(even.any(-1), even.argmax(-1), tied.argmax(-1))


def blocks(x):
    rows, cols = x.shape
    groups = -(-cols // 128)
    v = np.zeros((rows, groups * 128))
    v[:, :cols] = x
    return v.reshape(rows, groups * 4, 32)


def pack(fmt, x):
    """(codes, scales) of a float64 matrix; fmt "int8" or "fp4"."""
    v = blocks(np.asarray(x, np.float64))
    rows, nb, _ = v.shape
    bad = ~np.isfinite(v).all(2)
    v = np.where(bad[..., None], 0.0, v)
    a = np.abs(v).max(2)
    e = np.where(a > 0, np.frexp(a)[1] - 1, -127)
    e = np.maximum(e, -127)
    if fmt == "int8":
        scale = e + 127
        code = np.clip(np.rint(np.ldexp(v, 6 - e[..., None])), -127, 127).astype(np.int8)
        codes = code.reshape(rows, nb // 4, 128)
    else:
        scale = np.maximum(e - 2 + 127, 0)
        w = np.ldexp(v, 127 - scale[..., None])
        n = nearest_e2m1(np.abs(w)) + np.where(np.signbit(w), 8, 0)
        n = n.reshape(rows, nb // 4, 64, 2)
        codes = (n[..., 0] + 16 * n[..., 1]).astype(np.uint8)
    scale = np.where(bad, 255, scale)
    return codes, scale.astype(np.uint8).reshape(rows, nb // 4, 4)


def unpack(fmt, codes, scales, cols):
    rows = codes.shape[0]
    s = scales.reshape(rows, -1).astype(np.int64)
    if fmt == "int8":
        v = np.ldexp(codes.reshape(rows, -1, 32).astype(np.float64), (s - 133)[..., None])
    else:
        c = codes.reshape(rows, -1)
        n = np.stack([c & 15, c >> 4], 2).reshape(rows, -1, 32)
        v = np.ldexp(np.where(n & 8, -E2M1[n & 7], E2M1[n & 7]), (s - 127)[..., None])
    v = np.where((s == 255)[..., None], np.nan, v)
    return v.reshape(rows, -1)[:, :cols]


def kept(fmt, x):
    """What x reads as after packing."""
    return unpack(fmt, *pack(fmt, x), x.shape[1])


_erfc = np.vectorize(math.erfc, otypes=[np.float64])
C = math.sqrt(2 / math.pi)


def _logistic(z):
    with np.errstate(over="ignore"):
        return 1 / (1 + np.exp(-z))


def act(kind, x):
    """f(x); kind "gelu", "gelu_tanh" or "silu"."""
    if kind == "gelu":
        return 0.5 * x * _erfc(-x / math.sqrt(2))
    z = x if kind == "silu" else 2 * C * (x + 0.044715 * x ** 3)
    return x * _logistic(z)                           # (1 + tanh(z / 2)) / 2 without its loss near -1


def act_slope(kind, x):
    """f'(x)."""
    if kind == "gelu":
        return 0.5 * _erfc(-x / math.sqrt(2)) + x * np.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    z, dz = (x, 1.0) if kind == "silu" else (2 * C * (x + 0.044715 * x ** 3), 2 * C * (1 + 3 * 0.044715 * x * x))
    return _logistic(z) + x * _logistic(z) * _logistic(-z) * dz


def act_forward(kind, x, u=None):
    return act(kind, x) if u is None else act(kind, x) * u


def act_backward(kind, dy, x, u=None):
    """(dx, du) from packed and read back x (and u)."""
    xk = kept("int8", x)
    if u is None:
        return dy * act_slope(kind, xk), None
    return dy * act_slope(kind, xk) * kept("int8", u), dy * act(kind, xk)


def linear_forward(x, w, bias=None):
    """w: the packed weight's values."""
    y = kept("fp4", x) @ w.T
    return y if bias is None else y + bias


def linear_backward_input(dy, w):
    return dy @ w


def linear_backward_weight(dy, x, dw_in=None):
    """(dw, db)"""
    dw = dy.T @ kept("int8", x)
    return dw if dw_in is None else dw + dw_in, dy.sum(0)
