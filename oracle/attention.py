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


def visible(nq, nk, left, right, sinks):
    """bool [nq, nk]: which keys a query sees."""
    p = np.arange(nq)[:, None] + (nk - nq)
    j = np.arange(nk)[None, :]
    ok = np.ones((nq, nk), bool)
    if right >= 0:
        ok &= j <= p + right
    if left >= 0:
        ok &= (j >= p - left) | (j < sinks)
    return ok


def attention(q, k, v, q_lens, k_lens, left=-1, right=-1, sinks=0, scale=None):
    """q [Tq, H, D], k, v [Tk, Hk, D] float64 -> (out [Tq, H, D], lse [H, Tq]); what a query does not see is never read."""
    Tq, H, D = q.shape
    group = H // k.shape[1]
    scale = scale or 1.0 / np.sqrt(D)
    out, lse = np.zeros((Tq, H, D)), np.full((H, Tq), -np.inf)
    q0 = k0 = 0
    for nq, nk in zip(q_lens, k_lens):
        ok = visible(nq, nk, left, right, sinks)
        for h in range(H):
            kk, vv = k[k0:k0 + nk, h // group], v[k0:k0 + nk, h // group]
            for i in range(nq):
                see = ok[i]
                if not see.any():
                    continue
                with np.errstate(invalid="ignore", over="ignore"):
                    z = (kk[see] @ q[q0 + i, h]) * scale
                    m = z.max()
                    e = np.exp(z - m)
                    lse[h, q0 + i] = m + np.log(e.sum())
                    out[q0 + i, h] = (e @ vv[see]) / e.sum()
        q0, k0 = q0 + nq, k0 + nk
    return out, lse


def adapter_add(x, a, b, scale, lens, ids, base):
    """base + scale_i b_i (a_i x) segment by segment; ids outside the adapters leave base as it is."""
    y, at = np.array(base, np.float64), 0
    for n, i in zip(lens, ids):
        if 0 <= i < len(a):
            y[at:at + n] += scale[i] * ((x[at:at + n] @ a[i].T) @ b[i].T)
        at += n
    return y
