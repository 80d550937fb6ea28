"""The 64-bit definitions of embedding, norms between layers and the LM head's gradient, pinned against identities and differences (CPU)."""
import numpy as np
import pytest

from oracle import rows


def _slope(f, x, u, h=1e-5):
    return (f(x + h * u) - f(x - h * u)) / (2 * h)


def test_embedding_and_its_gradient_are_transposes():
    r = np.random.default_rng(0)
    tokens = np.array([3, -1, 0, 3, 7, 3, 6])
    table, dy = r.standard_normal((7, 8)), r.standard_normal((7, 8))
    out = rows.embed(tokens, table, 2.5)
    d, size = rows.embed_grad(tokens, dy, 7, 2.5)
    assert np.isclose((out * dy).sum(), (table * d).sum())
    assert (out[[1, 4]] == 0).all() and np.array_equal(out[0], 2.5 * table[3])
    assert np.allclose(d[3], 2.5 * (dy[0] + dy[3] + dy[5])) and (d[[1, 2, 4, 5]] == 0).all() and (size >= np.abs(d) - 1e-12).all()


@pytest.mark.parametrize("layer", [False, True])
def test_norm_and_its_gradient(layer):
    r = np.random.default_rng(1)
    x, dy, ds = r.standard_normal((3, 5, 24))
    w, b = 1 + 0.3 * r.standard_normal(24), r.standard_normal(24)
    n = rows.row_norm(x, layer, 1e-9)
    assert np.allclose((n * n).mean(-1), 1) and (not layer or np.allclose(n.mean(-1), 0))
    assert np.allclose(rows.row_norm(3 * x + (2 if layer else 0), layer, 1e-12), n, atol=1e-7)
    dx, dw, db = rows.row_norm_grad(dy, x, layer, 1e-3, w, ds)
    f = lambda x_, w_=w, b_=b: (rows.row_norm(x_, layer, 1e-3, w_, b_) * dy).sum() + (x_ * ds).sum()
    for _ in range(6):
        u, v = r.standard_normal(x.shape), r.standard_normal(24)
        assert np.isclose(_slope(f, x, u), (dx * u).sum(), rtol=1e-6, atol=1e-8)
        assert np.isclose(_slope(lambda q: f(x, q), w, v), (dw * v).sum(), rtol=1e-6, atol=1e-8)
        assert np.isclose(_slope(lambda q: f(x, w, q), b, v), (db * v).sum(), rtol=1e-6, atol=1e-8)


@pytest.mark.parametrize("inv_t,forbid", [(1.0, -1), (0.7, 4)])
def test_gradient_of_the_lm_head(inv_t, forbid):
    r = np.random.default_rng(2)
    h, w = r.standard_normal((4, 6)), r.standard_normal((11, 6))
    target, a, c = np.array([2, 10, -1, 0]), r.standard_normal(4), r.standard_normal(4)

    def outputs(h_, w_):
        z = h_ @ w_.T * inv_t
        zt = np.array([z[m, v] if v >= 0 else 0.0 for m, v in enumerate(target)])
        z = z if forbid < 0 else np.delete(z, forbid, 1)
        return np.log(np.exp(z).sum(1)), zt

    f = lambda h_, w_: (a * outputs(h_, w_)[0]).sum() + (c * outputs(h_, w_)[1]).sum()
    dz, dh, dw = rows.lmhead_grad(h, w, outputs(h, w)[0], a, c, target, inv_t, forbid)
    for _ in range(6):
        u, v = r.standard_normal(h.shape), r.standard_normal(w.shape)
        assert np.isclose(_slope(lambda q: f(q, w), h, u), (dh * u).sum(), rtol=1e-6, atol=1e-8)
        assert np.isclose(_slope(lambda q: f(h, q), w, v), (dw * v).sum(), rtol=1e-6, atol=1e-8)
    assert forbid < 0 or (dz[:, forbid] == 0).all()
    # a log-likelihood: every row's dz adds up to nothing
    dz, _, _ = rows.lmhead_grad(h, w, outputs(h, w)[0], -np.ones(4), np.ones(4), np.array([2, 10, 1, 0]), inv_t, forbid)
    assert np.allclose(dz.sum(1), 0)
