"""MXFP4 by its definition, in float64 on the CPU (numpy): what the kernels are compared with."""
import numpy as np

SIZES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantise(x):
    """x [rows][cols] -> (codes [rows][16 nb], scales [rows][nb]): element by element the nearest of the eight magnitudes, the
    even code where two are as near."""
    x = np.asarray(x)
    parts = [_quantise_rows(x[r:r + 256].astype(np.float64)) for r in range(0, x.shape[0], 256)]
    return np.concatenate([p[0] for p in parts]), np.concatenate([p[1] for p in parts])


def _quantise_rows(x):
    rows, cols = x.shape
    nb = (cols + 31) // 32
    b = np.zeros((rows, nb * 32))
    b[:, :cols] = x
    b = b.reshape(rows, nb, 32)
    bad = ~np.isfinite(b).all(axis=-1)
    b = np.where(bad[..., None], 0.0, b)
    top = np.abs(b).max(axis=-1)
    e = np.where(top > 0, np.clip(np.frexp(top)[1] - 3, -127, 127), -127)     # top = m 2^ex, m in [0.5, 1): ex - 1 - 2
    u = np.abs(b) / np.ldexp(1.0, e)[..., None]
    near, code = np.full(u.shape, np.inf), np.zeros(u.shape, dtype=np.uint8)
    for c in (0, 2, 4, 6, 1, 3, 5, 7):                                        # an even code keeps its place against an odd one as near
        far = np.abs(u - SIZES[c])
        code = np.where(far < near, c, code)
        near = np.minimum(near, far)
    code = np.where(bad[..., None], 0, code + 8 * np.signbit(b)).astype(np.uint8)
    code = code.reshape(rows, -1)
    return (code[:, 0::2] | code[:, 1::2] << 4).astype(np.uint8), np.where(bad, 255, e + 127).astype(np.uint8)


def values(codes, scales, cols):
    c = np.stack([codes & 15, codes >> 4], axis=-1).reshape(codes.shape[0], -1)
    v = SIZES[c & 7] * np.where(c & 8, -1.0, 1.0)
    s = np.ldexp(1.0, scales.astype(np.int64) - 127)
    s[scales == 255] = np.nan
    return (v.reshape(codes.shape[0], -1, 32) * s[..., None]).reshape(codes.shape[0], -1)[:, :cols]
