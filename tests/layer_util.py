"""Plain forms in 64 bits of a layer, its gradient and dropout, and how far
binary32 arithmetic and the roundings to a type may take a kernel from them."""
import math

import numpy as np
import torch

from tests.learn_util import TINY, UNIT

F32 = 2.0 ** -24                     # half a step of binary32, relative
M64 = (1 << 64) - 1
erfc = np.vectorize(math.erfc, otypes=[np.float64])


def mix(z):
    """SplitMix64's output function on numpy uint64."""
    z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
    z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
    return z ^ (z >> np.uint64(31))


def words(seed, count):
    with np.errstate(over="ignore"):
        key = mix(np.array([seed & M64], dtype=np.uint64))
        n = np.arange(1, count + 1, dtype=np.uint64)
        return mix(n * np.uint64(0x9E3779B97F4A7C15) + key)


def share(rows, cols, p, seed):
    """What the mask multiplies each element by, [rows, cols] float64."""
    if p == 0.0:
        return np.ones((rows, cols))
    pairs = (cols + 1) // 2
    w = words(seed, rows * pairs)
    bits = np.stack([w & np.uint64(0xFFFFFFFF), w >> np.uint64(32)], 1).reshape(rows, 2 * pairs)[:, :cols]
    keep = bits >= np.uint64(math.floor(p * 2 ** 32 + 0.5))
    return np.where(keep, 1.0 / (1.0 - p) if p < 1.0 else 0.0, 0.0)


def double(t):
    return t.detach().double().cpu().numpy()


def act(z, name):
    with np.errstate(over="ignore"):
        if name == "relu":
            return np.maximum(z, 0.0)
        if name == "gelu":
            return 0.5 * z * erfc(-z * math.sqrt(0.5))
        if name == "silu":
            return z / (1.0 + np.exp(-z))
    return z


def slope(z, name):
    with np.errstate(over="ignore"):
        if name == "relu":
            return (z > 0).astype(np.float64)
        if name == "gelu":
            return 0.5 * erfc(-z * math.sqrt(0.5)) + z * np.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
        if name == "silu":
            s = 1.0 / (1.0 + np.exp(-z))
            return s * (1.0 + z * (1.0 - s))
    return np.ones_like(z)


def half_step(v, dtype):
    return UNIT[dtype] * np.maximum(np.abs(v), TINY[dtype])


def product(a, b):
    """(a b^T, how far sums in binary32 may be off): every one of the terms'
    products and additions may lose a step of the sum of magnitudes, in whatever
    order; eight more for sums in parts."""
    return a @ b.T, 2 * F32 * (a.shape[1] + 8) * (np.abs(a) @ np.abs(b).T)


def layer(x, w, bias, name, residual, p, seed, dtype):
    """(y, its bound, z, its bound) of tensors, the result rounded to `dtype`."""
    z, off = product(double(x), double(w))
    if bias is not None:
        b = double(bias)[None, :]
        z, off = z + b, off + 2 * F32 * np.abs(b)
    off_z = off + 2 * F32 * np.abs(z)
    m = share(*z.shape, p, seed)
    y = m * act(z, name)
    # no activation is steeper than 1.13; its value is off by some steps of z (the exponent of exp
    # multiplies a step of z by |z|, which the value's own fall outweighs)
    off_y = m * (1.13 * off_z + 16 * F32 * np.abs(z))
    if residual is not None:
        y = y + double(residual)
    off_y = off_y + 8 * F32 * np.abs(y)
    return y, off_y + half_step(np.abs(y) + off_y, dtype), z, off_z + half_step(np.abs(z) + off_z, x.dtype)


def gradients(grad, x, w, pre, name, p, seed):
    """((dx, bound), (dw, bound), (db, bound in float32)) from tensors."""
    dy, x64, w64 = double(grad), double(x), double(w)
    m = share(*dy.shape, p, seed)
    kept = (m > 0).astype(np.float64)
    s = 1.0 if p == 0.0 or p == 1.0 else 1.0 / (1.0 - p)
    before = kept * dy
    off = np.zeros_like(before)
    if name is not None:
        z = double(pre)
        before = before * slope(z, name)
        off = kept * np.abs(dy) * 32 * F32 * (1.0 + np.abs(z)) if name != "relu" else off
    db = s * before.sum(0)
    off_db = s * (off.sum(0) + 2 * F32 * (len(dy) + 8) * np.abs(before).sum(0)) + 4 * F32 * np.abs(db)
    # dz as the products take it, rounded to x's type before its share
    off = off + half_step(np.abs(before) + off, x.dtype)
    out = []
    for a, b, off_a in ((before, w64.T, off), (before.T, x64.T, off.T)):
        v, off_v = product(a, b)
        off_v = s * (off_v + off_a @ np.abs(b).T) + 4 * F32 * s * np.abs(v)
        v = s * v
        out.append((v, off_v + half_step(np.abs(v) + off_v, x.dtype)))
    return out[0], out[1], (db, off_db)


def assert_within(got, want, bound, what=""):
    g = double(got)
    assert g.shape == want.shape, (what, g.shape, want.shape)
    bad = ~(np.abs(g - want) <= bound)
    if bad.any():
        at = tuple(int(k[0]) for k in np.nonzero(bad))
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.size}, first at {at}: {g[at]} for {want[at]} within {bound[at]}")
