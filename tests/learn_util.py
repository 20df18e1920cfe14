"""Plain forms in 64 bits of the operators on learned tables and layers, and
the error that rounding their results to a type allows."""
import numpy as np
import torch

# half the spacing of a type's numbers relative to them, and its smallest normal number
UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -126, torch.float16: 2.0 ** -14, torch.bfloat16: 2.0 ** -126}


def rounding(want, dtype):
    """Most that rounding `want` (float64) to dtype moves it."""
    return UNIT[dtype] * np.maximum(np.abs(want), TINY[dtype])


def infinite(want, dtype):
    """`want` with infinities where rounding to dtype makes them."""
    with np.errstate(over="ignore"):
        big = torch.from_numpy(want).to(dtype).double().numpy()
    return np.where(np.isinf(big), big, want)


def gradient(grad, ids, rows, scale):
    """(scale sum of the rows of each index, the sum of magnitudes, the counts) in float64."""
    g = grad.double().cpu().numpy().reshape(-1, grad.shape[-1])
    v = ids.cpu().numpy().reshape(-1)
    total, size = np.zeros((rows, g.shape[1])), np.zeros((rows, g.shape[1]))
    ok = (v >= 0) & (v < rows)
    np.add.at(total, v[ok], g[ok])
    np.add.at(size, v[ok], np.abs(g[ok]))
    s = float(np.float32(scale))
    return s * total, abs(s) * size, np.bincount(v[ok], minlength=rows)[:, None]


def newton_schulz(g, steps, coefficients, eps):
    a, b, c = (float(np.float32(k)) for k in coefficients)
    x = g.double().cpu().numpy()
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x
    norm = np.sqrt((x * x).sum()) + float(np.float32(eps))
    x = x / norm if norm > 0 else x
    for _ in range(steps):
        p = x @ x.T
        x = a * x + (b * p + c * (p @ p)) @ x
    return x.T if tall else x


MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantise(x):
    """(codes [rows, blocks 16], scales [rows, blocks], values [rows, cols]) of
    x [rows, cols], from the definition: the nearest of the eight magnitudes,
    the even code in a tie."""
    v = x.double().cpu().numpy()
    rows, cols = v.shape
    blocks = -(-cols // 32)
    full = np.zeros((rows, blocks * 32))
    full[:, :cols] = v
    full = full.reshape(rows, blocks, 32)
    bad = ~np.isfinite(full).all(axis=2)
    clean = np.where(bad[:, :, None], 0.0, full)
    top = np.abs(clean).max(axis=2)
    _, e = np.frexp(top)                               # top = f 2^e with f in [0.5, 1)
    e = np.where(top > 0, np.maximum(e - 3, -127), -127)
    u = np.abs(clean) / np.ldexp(1.0, e)[:, :, None]
    far = np.abs(u[..., None] - MAGNITUDES)
    near = far.min(axis=3, keepdims=True) == far
    # of two that are equally near, the even one
    code = np.where(near & (np.arange(8) % 2 == 0), 16, 0) + np.where(near, 1, 0)
    code = code.argmax(axis=3)
    value = MAGNITUDES[code] * np.ldexp(1.0, e)[:, :, None]
    value = np.where(np.signbit(clean), -value, value)
    value = np.where(bad[:, :, None], np.nan, value).reshape(rows, -1)[:, :cols]
    code = np.where(np.signbit(clean), code + 8, code).reshape(rows, -1, 2).astype(np.uint8)
    scales = np.where(bad, 255, e + 127).astype(np.uint8)
    return code[..., 0] | code[..., 1] << 4, scales, value
