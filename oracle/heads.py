"""Head norms with rotation, their gradient, and attention over a paged cache, in 64 bits with numpy: definitions written out, one row at a time
where that is simplest.  Test infrastructure."""
import numpy as np


def e4m3_values():
    """What each of the 256 codes stands for: sign, 4 exponent bits (bias 7), 3 mantissa bits; code 0x7f is NaN, nothing is infinite."""
    v = np.empty(256)
    for code in range(256):
        e, m = (code >> 3) & 15, code & 7
        x = np.nan if (code & 0x7f) == 0x7f else (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
        v[code] = -x if code & 0x80 else x
    return v


def e4m3_distance(x):
    """Distance from each x to the nearest finite e4m3 value (beyond 448: to 448)."""
    pos = np.sort(e4m3_values()[:127])
    a = np.abs(np.asarray(x, dtype=np.float64))
    i = np.clip(np.searchsorted(pos, a), 1, len(pos) - 1)
    return np.minimum(np.abs(a - pos[i - 1]), np.abs(a - pos[i]))


def angles(n_pos, rot, theta=10000.0):
    """fp64 [n_pos, rot]: cosines, then sines, of p theta^(-2 i / rot)."""
    a = np.arange(n_pos)[:, None] * theta ** (-np.arange(0, rot, 2) / rot)
    return np.concatenate([np.cos(a), np.sin(a)], axis=1)


def _pairs(d, rot, style):
    """Indices of the first and second entry of every rotated pair (style 0: halves, 1: neighbours)."""
    i = np.arange(rot // 2)
    return (i, i + rot // 2) if style == 0 else (2 * i, 2 * i + 1)


def rotate(x, table, positions, style, back=False):
    """x [T, H, d]; table [n, rot] (cosines, sines) or None."""
    if table is None:
        return x.copy()
    rot = table.shape[1]
    i, j = _pairs(x.shape[-1], rot, style)
    c, s = table[positions, None, :rot // 2], table[positions, None, rot // 2:]
    if back:
        s = -s
    y = x.copy()
    y[..., i], y[..., j] = x[..., i] * c - x[..., j] * s, x[..., j] * c + x[..., i] * s
    return y


def head_map(x, w, eps, table, positions, style):
    if w is not None:
        x = x * w / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return rotate(x, table, positions, style)


def head_map_grad(dy, x, w, eps, table, positions, style):
    """(dx, dw) for the upstream gradient dy; dw is None without a weight."""
    dz = rotate(dy, table, positions, style, back=True)
    if w is None:
        return dz, None
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    n, g = x * r, dz * w
    return r * (g - n * (g * n).mean(-1, keepdims=True)), (dz * n).sum((0, 1))


def paged_rows(pages, table_row, n):
    """Rows 0 .. n - 1 of a sequence [n, Hkv, d] from pages [n_pages, Hkv, page_size, d], and which of them exist."""
    page_size = pages.shape[2]
    got, there = np.zeros((n, pages.shape[1], pages.shape[3])), np.zeros(n, dtype=bool)
    for t in range(n):
        page = int(table_row[t // page_size])
        if 0 <= page < pages.shape[0]:
            got[t], there[t] = pages[page, :, t % page_size], True
    return got, there


def paged_attention(q, pages_k, pages_v, table, kv_len, q_len=None, block_size=0, scale=None):
    """q [B, Lq, Hq, d].  Returns out, lse, and what bounds of the error are made of: A = sum_j p_j |v_j| like out, and S = the largest scaled
    score sum |q||k| of the row like lse; rows behind q_len are NaN."""
    B, Lq, Hq, d = q.shape
    g = Hq // pages_k.shape[1]
    scale = d ** -0.5 if scale is None else scale
    out, mag = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    lse, top = np.full((B, Hq, Lq), np.nan), np.full((B, Hq, Lq), np.nan)
    for b in range(B):
        n, ql = int(kv_len[b]), Lq if q_len is None else int(q_len[b])
        k, there = paged_rows(pages_k, table[b], n)
        v, _ = paged_rows(pages_v, table[b], n)
        for i in range(ql):
            seen = there.copy()
            if block_size:
                seen &= np.arange(n) // block_size <= (n - ql + i) // block_size
            for h in range(Hq):
                kk, vv = k[seen, h // g], v[seen, h // g]
                if not len(kk):
                    out[b, i, h], mag[b, i, h], lse[b, h, i], top[b, h, i] = 0, 0, -np.inf, 0
                    continue
                s = kk @ q[b, i, h] * scale
                m = s.max()
                p = np.exp(s - m)
                lse[b, h, i] = m + np.log(p.sum())
                p /= p.sum()
                out[b, i, h], mag[b, i, h] = p @ vv, p @ np.abs(vv)
                top[b, h, i] = (np.abs(kk) @ np.abs(q[b, i, h])).max() * scale
    return out, lse, mag, top
