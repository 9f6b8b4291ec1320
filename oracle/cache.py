"""Plain fp64 form of the paged cache of quantized keys and values: elements by search among all values of the format, one group, token
and query at a time.  Everything is written from the definitions."""
import numpy as np

from . import attention as oat

BITS = {"fp8": 8, "fp4": 4}
MAX_EXP = {"fp8": 7, "fp4": 13}
MIN_EXP, BROKEN = -14, 255


def values(kind):
    """float64 value of every element code (the two NaN codes of e4m3 as NaN)."""
    out = []
    m_bits, bias, e_max = (3, 7, 15) if kind == "fp8" else (1, 1, 3)
    for code in range(1 << BITS[kind]):
        sign = -1.0 if code >> (BITS[kind] - 1) else 1.0
        e, m = (code >> m_bits) & e_max, code & ((1 << m_bits) - 1)
        if kind == "fp8" and e == 15 and m == 7:
            out.append(np.nan)
        elif e:
            out.append(sign * (1 + m / 2.0 ** m_bits) * 2.0 ** (e - bias))
        else:
            out.append(sign * (m / 2.0 ** m_bits) * 2.0 ** (1 - bias))
    return np.array(out)


def encode(x, kind):
    """x float64 [..., D] (finite) -> (codes [..., D], scale bytes [..., D / 32])."""
    v = values(kind)
    half = 1 << (BITS[kind] - 1)
    grid = v[:half - 1] if kind == "fp8" else v[:half]                    # magnitudes, ascending, without NaN
    g = np.asarray(x, np.float64).reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    top = np.abs(g).max(-1)
    k = np.full(top.shape, MIN_EXP)
    for e in range(MIN_EXP, MAX_EXP[kind]):
        k[top > grid[-1] * 2.0 ** e] = e + 1
    a = np.minimum(np.abs(g) * 2.0 ** -k[..., None].astype(np.float64), grid[-1])
    hi = np.searchsorted(grid, a)                                         # grid[hi - 1] < a <= grid[hi]
    lo = np.maximum(hi - 1, 0)
    up = grid[hi] - a
    down = a - grid[lo]
    code = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))      # ties: the even code
    return (code + half * np.signbit(g)).reshape(x.shape), (k + 127).astype(np.uint8)


def decode(codes, scales, kind):
    y = values(kind)[codes].reshape(*codes.shape[:-1], codes.shape[-1] // 32, 32)
    s = np.where(scales == BROKEN, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return (y * s[..., None]).reshape(codes.shape)


def block_bytes(page, d, kind):
    return 2 * page * (d * BITS[kind] // 8 + d // 32)


def _parts(block, page, d, kind):
    """Views of a block's (keys, values, scales of keys, of values), one row a token."""
    row, groups = d * BITS[kind] // 8, d // 32
    ends = np.cumsum([0, page * row, page * row, page * groups, page * groups])
    return [block[a:b].reshape(page, -1) for a, b in zip(ends, ends[1:])]


def places(table, lens, page, n_pages, seq, n):
    """(page or -1, token of it) of the last n positions of a sequence; -2 before its beginning."""
    end = min(max(int(lens[seq]), 0), table.shape[1] * page)
    out = []
    for p in range(end - n, end):
        if p < 0:
            out.append((-2, 0))
        else:
            at = int(table[seq, p // page])
            out.append((at if 0 <= at < n_pages else -1, p % page))
    return out


def write(pages, k, v, table, lens, new, d, kind, first=0):
    """pages uint8 [n, heads, block bytes] (changed in place); k, v float64 [T, heads, d]; new: tokens of each sequence."""
    n_pages, heads, size = pages.shape
    page = size // (block_bytes(1, d, kind))
    fine = np.isfinite(k).all(-1) & np.isfinite(v).all(-1)
    (k_code, k_scale), (v_code, v_scale) = (encode(np.where(fine[..., None], x, 0.0), kind) for x in (k, v))
    t = first
    for s, n in enumerate(new):
        for at, tok in places(table, lens, page, n_pages, s, n):
            if at >= 0:
                for h in range(heads):
                    parts = _parts(pages[at, h], page, d, kind)
                    for i, code, scale in ((0, k_code[t, h], k_scale[t, h]), (1, v_code[t, h], v_scale[t, h])):
                        parts[i][tok] = code if kind == "fp8" else code[0::2] | code[1::2] << 4
                        parts[2 + i][tok] = scale if fine[t, h] else BROKEN
            t += 1


def read(pages, table, lens, new, d, kind):
    """(K, V) float64 [T, heads, d], and bool [T]: a page holds the token.  Zeros where none does."""
    n_pages, heads, size = pages.shape
    page = size // (block_bytes(1, d, kind))
    total = sum(new)
    raw = np.zeros((2, total, heads, d * BITS[kind] // 8), np.uint8)
    scales = np.full((2, total, heads, d // 32), 127, np.uint8)
    here = np.zeros(total, bool)
    t = 0
    for s, n in enumerate(new):
        for at, tok in places(table, lens, page, n_pages, s, n):
            if at >= 0:
                here[t] = True
                for h in range(heads):
                    parts = _parts(pages[at, h], page, d, kind)
                    for i in range(2):
                        raw[i, t, h], scales[i, t, h] = parts[i][tok], parts[2 + i][tok]
            t += 1
    code = raw if kind == "fp8" else np.stack((raw & 15, raw >> 4), -1).reshape(2, total, heads, d)
    out = decode(code.astype(np.int64), scales, kind)
    return out[0], out[1], here


def attention(q, pages, table, lens, new, kind, left=-1, right=0, sinks=0, scale=None):
    """q float64 [T, H, D] -> (out [T, H, D], lse [H, T], sum of weights times |v|); what a query does not see is never used."""
    T, H, D = q.shape
    group = H // pages.shape[1]
    page = pages.shape[2] // block_bytes(1, D, kind)
    scale = scale or 1.0 / np.sqrt(D)
    out, lse, size = np.zeros((T, H, D)), np.full((H, T), -np.inf), np.zeros((T, H, D))
    t0 = 0
    for s, n in enumerate(new):
        nk = min(max(int(lens[s]), 0), table.shape[1] * page)
        k, v, here = read(pages, table[s:s + 1], [nk], [nk], D, kind)
        ok = oat.visible(n, nk, left, right, sinks) & here[None]
        for i in range(n):
            seen = np.flatnonzero(ok[i])
            if not seen.size:
                continue
            for h in range(H):
                if not np.isfinite(q[t0 + i, h]).all() or np.isnan(k[seen, h // group]).any():
                    out[t0 + i, h] = lse[h, t0 + i] = size[t0 + i, h] = np.nan
                    continue
                z = scale * (k[seen, h // group] @ q[t0 + i, h])
                m = z.max()
                w = np.exp(z - m)
                lse[h, t0 + i] = m + np.log(w.sum())
                w /= w.sum()
                out[t0 + i, h] = w @ v[seen, h // group]
                size[t0 + i, h] = w @ np.abs(v[seen, h // group])
        t0 += n
    return out, lse, size
