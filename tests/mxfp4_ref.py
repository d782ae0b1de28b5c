"""MXFP4 by its definition, in float64 on the CPU (numpy): what the kernels are compared with."""
import numpy as np

SIZES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantise(x):
    """x [rows][cols] -> (codes [rows][16 nb], scales [rows][nb]): element by element the nearest of the eight magnitudes, the
    even code where two are as near."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    nb = (cols + 31) // 32
    b = np.zeros((rows, nb * 32))
    b[:, :cols] = x
    b = b.reshape(rows, nb, 32)
    bad = ~np.isfinite(b).all(axis=-1)
    b = np.where(bad[..., None], 0.0, b)
    top = np.abs(b).max(axis=-1)
    e = np.full(top.shape, -127, dtype=np.int64)
    for i in np.argwhere(top > 0):
        m, ex = np.frexp(top[tuple(i)])          # top = m 2^ex, m in [0.5, 1)
        e[tuple(i)] = max(-127, min(127, ex - 1 - 2))
    u = np.abs(b) / np.ldexp(1.0, e)[..., None]
    far = np.abs(u[..., None] - SIZES)
    near = far.min(axis=-1, keepdims=True)
    # lowest even code among the nearest, else the lowest
    order = np.array([0, 2, 4, 6, 1, 3, 5, 7])
    code = order[(far == near)[..., order].argmax(axis=-1)].astype(np.uint8)
    code = np.where(bad[..., None], 0, code + 8 * np.signbit(b)).astype(np.uint8)
    code = code.reshape(rows, -1)
    return (code[:, 0::2] | code[:, 1::2] << 4).astype(np.uint8), np.where(bad, 255, e + 127).astype(np.uint8)


def values(codes, scales, cols):
    c = np.stack([codes & 15, codes >> 4], axis=-1).reshape(codes.shape[0], -1)
    v = SIZES[c & 7] * np.where(c & 8, -1.0, 1.0)
    s = np.ldexp(1.0, scales.astype(np.int64) - 127)
    s[scales == 255] = np.nan
    return (v.reshape(codes.shape[0], -1, 32) * s[..., None]).reshape(codes.shape[0], -1)[:, :cols]
