"""The 64-bit definitions of head norms, rotation, e4m3 and paged attention, pinned against identities and differences (CPU)."""
import numpy as np
import pytest
import torch

import oracle
from oracle import heads


def _case(seed, T=5, H=3, d=64, rot=64, norm=True):
    r = np.random.default_rng(seed)
    x, dy = r.standard_normal((2, T, H, d))
    return x, dy, (1 + 0.3 * r.standard_normal(d)) if norm else None, heads.angles(40, rot) if rot else None, r.integers(0, 40, T)


def test_e4m3_codes_are_torchs():
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(codes, heads.e4m3_values(), equal_nan=True)
    x = np.array([0.0, 2.0 ** -10, 3.1, -3.1, 448.0, 500.0])
    assert np.allclose(heads.e4m3_distance(x), [0, 2.0 ** -10, 0.1, 0.1, 0, 52])


@pytest.mark.parametrize("style", [0, 1])
@pytest.mark.parametrize("rot", [16, 48, 64])
def test_rotation_keeps_lengths_and_depends_on_differences(style, rot):
    x, y, _, table, pos = _case(3, rot=rot)
    a = heads.rotate(x, table, pos, style)
    assert np.allclose(np.linalg.norm(a, axis=-1), np.linalg.norm(x, axis=-1))
    assert np.array_equal(a[..., rot:], x[..., rot:])
    assert np.allclose(heads.rotate(a, table, pos, style, back=True), x)
    one = np.ones(5, dtype=int)         # scores depend on the difference of positions only
    score = lambda m, n: (heads.rotate(x, table, m * one, style) * heads.rotate(y, table, n * one, style)).sum(-1)
    assert np.allclose(score(3, 9), score(20, 26))


@pytest.mark.parametrize("style,rot,norm", [(0, 64, True), (1, 32, True), (0, 0, True), (1, 64, False)])
def test_gradient_against_differences(style, rot, norm):
    x, dy, w, table, pos = _case(5, rot=rot, norm=norm)
    f = lambda x_, w_: (heads.head_map(x_, w_, 1e-3, table, pos, style) * dy).sum()
    dx, dw = heads.head_map_grad(dy, x, w, 1e-3, table, pos, style)
    r, h = np.random.default_rng(1), 1e-5
    for _ in range(8):
        u = r.standard_normal(x.shape)
        assert np.isclose((f(x + h * u, w) - f(x - h * u, w)) / (2 * h), (dx * u).sum(), rtol=1e-6, atol=1e-8)
    if norm:
        u = r.standard_normal(w.shape)
        assert np.isclose((f(x, w + h * u) - f(x, w - h * u)) / (2 * h), (dw * u).sum(), rtol=1e-6, atol=1e-8)
    else:
        assert dw is None


@pytest.mark.parametrize("block_size", [0, 1, 4])
def test_paged_attention_is_the_dense_one(block_size):
    """Pages in any order hold a dense cache; the dense oracle gives the same rows, and a page that is absent its keys' absence."""
    r = np.random.default_rng(7)
    B, Lq, Hq, Hkv, d, page, n = 2, 3, 4, 2, 64, 16, 37
    q, k, v = r.standard_normal((B, Lq, Hq, d)), r.standard_normal((B, n, Hkv, d)), r.standard_normal((B, n, Hkv, d))
    order = r.permutation(8)
    table = order[:6].reshape(2, 3)
    pk, pv = np.full((2, 8, Hkv, page, d), np.nan)
    for b in range(B):
        for t in range(n):
            pk[table[b, t // page], :, t % page], pv[table[b, t // page], :, t % page] = k[b, t], v[b, t]
    out, lse, mag, _ = heads.paged_attention(q, pk, pv, table, [n, n], block_size=block_size)
    for b in range(B):
        for i in range(Lq):
            m = n if not block_size else min(n, ((n - Lq + i) // block_size + 1) * block_size)
            for h in range(Hq):
                s = k[b, :m, h // 2] @ q[b, i, h] / 8
                p = np.exp(s) / np.exp(s).sum()
                assert np.allclose(out[b, i, h], p @ v[b, :m, h // 2]) and np.isclose(lse[b, h, i], np.log(np.exp(s).sum()))
                assert (mag[b, i, h] >= np.abs(out[b, i, h]) - 1e-12).all()
    table[0, 0] = -1
    out, lse, _, _ = heads.paged_attention(q, pk, pv, table, [n, 16], q_len=[3, 2])
    s = k[0, 16:, 0] @ q[0, 0, 0] / 8
    assert np.isclose(lse[0, 0, 0], np.log(np.exp(s).sum())) and np.isnan(out[1, 2]).all()
    out, lse, _, _ = heads.paged_attention(q, pk, pv, table, [16, 0])
    assert (out == 0).all() and (lse == -np.inf).all()
    assert oracle.heads is heads
