"""Embedding, the norms between layers and the LM head's gradient, in 64 bits with numpy: definitions written out.  Test infrastructure."""
import numpy as np


def embed(tokens, table, scale):
    out = np.zeros((len(tokens), table.shape[1]))
    for t, x in enumerate(tokens):
        if 0 <= x < len(table):
            out[t] = scale * table[x]
    return out


def embed_grad(tokens, dy, V, scale):
    """(gradient, the sum of the sizes that each of its entries is added up from)"""
    d, size = np.zeros((2, V, dy.shape[1]))
    live = (tokens >= 0) & (tokens < V)
    np.add.at(d, tokens[live], scale * dy[live])
    np.add.at(size, tokens[live], np.abs(scale * dy[live]))
    return d, size


def normalise(x, layer, eps):
    """(normalised rows, their factors)"""
    if layer:
        x = x - x.mean(-1, keepdims=True)
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return x * r, r


def row_norm(x, layer, eps, w=None, b=None):
    y, _ = normalise(x, layer, eps)
    if w is not None:
        y = y * w
    return y if b is None else y + b


def row_norm_grad(dy, x, layer, eps, w=None, ds=None):
    """(d_x, d_weight, d_bias)"""
    n, r = normalise(x, layer, eps)
    g = dy if w is None else dy * w
    dx = g - n * (g * n).mean(-1, keepdims=True)
    if layer:
        dx = dx - g.mean(-1, keepdims=True)
    dx = dx * r
    return dx if ds is None else dx + ds, (dy * n).sum(0), dy.sum(0)


def lmhead_grad(h, w, lse, d_lse, d_zt, target, inv_t=1.0, forbid=-1):
    """(dz, d_hidden, d_w) of sum(d_lse lse) + sum(d_zt ztarget), with p = exp(z - lse) from the lse that is given; d_lse, d_zt, target may be None."""
    p = np.exp(h @ w.T * inv_t - lse[:, None])
    if forbid >= 0:
        p[:, forbid] = 0.0
    dz = np.zeros_like(p)
    if d_lse is not None:
        live = d_lse != 0
        dz[live] = d_lse[live, None] * p[live]
    if d_zt is not None:
        for m, v in enumerate(target):
            if 0 <= v < len(w) and v != forbid:
                dz[m, v] += d_zt[m]
    dz *= inv_t
    return dz, dz @ w, dz.T @ h
