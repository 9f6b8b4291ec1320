"""Plain fp64 forms of the operators around the quantized projections: norms of queries and keys with their rotation by
position, windowed attention, low-rank adapters.  Everything is written from the definitions, one loop per head, sequence
or segment; inputs are float64 arrays."""
import numpy as np


def rope_angles(pos, axis_dims, theta):
    """float64 [T, sum(axis_dims) / 2]: pos[t, a] * theta^(-2 i / d_a), the axes' pairs one after the other."""
    cols = []
    for a, d in enumerate(axis_dims):
        freq = np.array([theta ** (-2.0 * i / d) for i in range(d // 2)])
        cols.append(pos[:, a, None].astype(np.float64) * freq[None, :])
    return np.concatenate(cols, axis=1)


def norm_rope(x, w, norm, eps, pos=None, axis_dims=(), theta=1.0, layout="pairs"):
    """x [T, H, D] -> normed (norm: "none", "head", "row") and turned."""
    x = np.asarray(x, np.float64)
    T, H, D = x.shape
    if norm == "head":
        x = x / np.sqrt((x ** 2).mean(axis=2, keepdims=True) + eps)
    elif norm == "row":
        x = x / np.sqrt((x ** 2).mean(axis=(1, 2), keepdims=True) + eps)
    if w is not None:
        x = x * (w[None, None, :] if norm == "head" else w.reshape(1, H, D))
    if pos is None:
        return x
    ang = rope_angles(pos, axis_dims, theta)
    y, at = x.copy(), 0
    for d in axis_dims:
        for i in range(d // 2):
            lo, hi = (at + 2 * i, at + 2 * i + 1) if layout == "pairs" else (at + i, at + d // 2 + i)
            c, s = np.cos(ang[:, at // 2 + i])[:, None], np.sin(ang[:, at // 2 + i])[:, None]
            y[:, :, lo] = x[:, :, lo] * c - x[:, :, hi] * s
            y[:, :, hi] = x[:, :, lo] * s + x[:, :, hi] * c
        at += d
    return y
