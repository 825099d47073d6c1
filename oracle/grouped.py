"""CPU oracle of the weights with group scales, their products and the norm, in numpy: written from the definitions in
include/skim.h, one plain loop or expression each, sums in binary64.  Test infrastructure only."""
import numpy as np


def _f32(v):
    return np.asarray(v, dtype=np.float32)


def quantize(w, group, r=None):
    """(codes, scales binary16, zero points) of a float16 matrix; r: reciprocal scale vector, float32."""
    x = _f32(w) if r is None else _f32(w) * _f32(r)
    rows, cols = x.shape
    groups = -(-cols // group)
    codes = np.zeros((rows, cols), np.int64)
    scale = np.zeros((rows, groups), np.float16)
    zero = np.zeros((rows, groups), np.int64)
    for k in range(groups):
        part = x[:, k * group:(k + 1) * group]
        low = np.minimum(part.min(axis=1), np.float32(0))
        high = np.maximum(part.max(axis=1), np.float32(0))
        s = (_f32(high - low) / np.float32(15)).astype(np.float16)
        by = np.where(s > 0, s, 1).astype(np.float64)
        z = np.clip(np.rint(-low.astype(np.float64) / by), 0, 15)
        q = np.clip(np.rint(part.astype(np.float64) / by[:, None]) + z[:, None], 0, 15)
        some = s > 0
        scale[:, k] = s
        zero[:, k] = np.where(some, z, 0)
        codes[:, k * group:(k + 1) * group] = np.where(some[:, None], q, 0)
    return codes, scale, zero


def values(codes, scale, zero, group):
    """The binary64 matrix that the codes stand for."""
    at = np.arange(codes.shape[1]) // group
    return (codes - zero[:, at]).astype(np.float64) * scale.astype(np.float64)[:, at]


def store(codes, scale, zero, group):
    """The stored form, byte by byte as declared."""
    rows, cols = codes.shape
    rt, ct, per = -(-rows // 16), -(-cols // 128), 128 // group
    record = 256 + 16 * per
    out = np.zeros((rt, ct, record), np.uint32)
    for i in range(rows):
        for j in range(cols):
            c, inside = divmod(j, 128)
            t, rest = divmod(inside, 32)
            p, e = divmod(rest, 8)
            out[i // 16, c, 16 * (i % 16) + 4 * p + t] |= np.uint32(int(codes[i, j]) << (4 * (4 * (e & 1) + e // 2)))
        for k in range(scale.shape[1]):
            c, inside = divmod(k, per)
            out[i // 16, c, 256 + (i % 16) * per + inside] = int(scale[i, k].view(np.uint16)) | int(zero[i, k]) << 16
    return out.reshape(-1).view(np.uint8)


def error(w, value, importance=None, r=None):
    x = _f32(w) if r is None else _f32(w) * _f32(r)
    d = (x.astype(np.float64) - value) ** 2
    return (d if importance is None else d * importance.astype(np.float64)).sum(axis=1)


def product(value, x, x_scale=None):
    """(x value^T, sum of the terms' magnitudes), rows of x times x_scale."""
    x = x.astype(np.float64)
    if x_scale is not None:
        x = x * x_scale.astype(np.float64)[:, None]
    return x @ value.T, np.abs(x) @ np.abs(value).T


def activation(name, g):
    if name == "silu":
        return g / (1.0 + np.exp(-g))
    return 0.5 * g * (1.0 + np.tanh(np.sqrt(2.0 / np.pi) * (g + 0.044715 * g ** 3)))


def add_rmsnorm(x, residual, weight, eps):
    """(h, p * rstd, codes, scale): x, residual, weight float32 arrays holding the 16-bit values."""
    h32 = _f32(x) if residual is None else _f32(x) + _f32(residual)
    h = x.astype(np.float64) if residual is None else x.astype(np.float64) + residual.astype(np.float64)
    w = np.ones(x.shape[1], np.float32) if weight is None else _f32(weight)
    rstd = 1.0 / np.sqrt((h * h).mean(axis=1) + eps)
    p = (h32 * w).astype(np.float64)
    a = np.abs(p).max(axis=1)
    codes = np.rint(127.0 * p / np.where(a > 0, a, 1.0)[:, None]).astype(np.int64)
    return h, h * w.astype(np.float64) * rstd[:, None], codes, a * rstd / 127.0
