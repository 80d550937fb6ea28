"""Head norms with rotation, their gradient and the append into a paged cache against the 64-bit definitions (GPU).

Bounds, u = 2^-24 (half a step of fp32), h = 2^-8 (half a step of bf16).  The norm's factor is a sum of d squares, a division, a root: relative error
under (d/2 + 8) u <= 72 u; two products more; a rotated entry is the sum of two such terms, at most sqrt(2) times the pair's length, the table's entries
rounded to fp32 in both.  Together under 128 u of the pair's length, then one rounding to bf16.  Gradients: sums of d products of two such numbers twice
over, under 400 u of what is added up."""
import numpy as np
import pytest
import torch

from oracle import heads
from paper_2604_04215_amd import binding as dlm
from gpu_util import DEV

pytestmark = pytest.mark.gpu
U, H = 2.0 ** -24, 2.0 ** -8
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32
EPS = 1e-6


def wide(t):
    return t.detach().double().cpu().numpy()


def bf16(rng, *shape, std=1.0):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32) * std).to(BF16).to(DEV)


class Case:
    def __init__(self, T, Hq, Hkv, d, rot, style=0, norm=True, seed=0, packed=True, n_pos=50):
        rng = self.rng = np.random.default_rng(1000 * T + 10 * Hq + d + rot + seed)
        x = bf16(rng, T, Hq + 2 * Hkv, d) if packed else bf16(rng, Hq + 2 * Hkv, T, d).transpose(0, 1)       # token-major or head-major
        self.T, self.Hq, self.Hkv, self.d, self.style = T, Hq, Hkv, d, style
        self.q, self.k, self.v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
        self.w = [(1 + 0.2 * bf16(rng, d).float()).to(BF16) for _ in range(2)] if norm else [None, None]
        self.pos = torch.from_numpy(rng.integers(0, n_pos, T).astype(np.int32)).to(DEV)
        self.rope = torch.from_numpy(heads.angles(n_pos, rot).astype(np.float32)).to(DEV) if rot else None

    def how(self):
        return dict(q_weight=self.w[0], k_weight=self.w[1], eps=EPS, rope=self.rope, positions=self.pos, rope_style=self.style)

    def table(self):
        return None if self.rope is None else wide(self.rope)

    def want(self, x, w):
        """(y, the length of each entry's pair before the rotation)"""
        x, pos = wide(x), self.pos.cpu().numpy()
        w = None if w is None else wide(w)
        y = heads.head_map(x, w, EPS, self.table(), pos, self.style)
        z = heads.head_map(x, w, EPS, None, None, 0)
        size = np.abs(z)
        if self.rope is not None:
            i, j = heads._pairs(self.d, self.rope.shape[1], self.style)
            size[..., i] = size[..., j] = np.hypot(z[..., i], z[..., j])
        return y, size


def check_heads(got, y, size):
    err = np.abs(wide(got) - y)
    assert (err <= H * np.abs(y) * (1 + H) + 128 * U * size * (1 + H) + 2.0 ** -133).all(), (err / (np.abs(y) + 1e-30)).max()


SHAPES = [(1, 1, 1, 64, 64), (1, 32, 8, 128, 128), (3, 4, 4, 64, 32), (5, 14, 2, 64, 64), (37, 28, 4, 128, 64), (64, 32, 8, 128, 128), (131, 3, 1, 128, 16),
          (257, 7, 7, 64, 48), (1030, 5, 2, 128, 112), (33, 9, 3, 128, 0)]


@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("style", [dlm.ROPE_HALVES, dlm.ROPE_PAIRS])
@pytest.mark.parametrize("T,Hq,Hkv,d,rot", SHAPES)
def test_forward(T, Hq, Hkv, d, rot, style, norm):
    c = Case(T, Hq, Hkv, d, rot, style, norm)
    qo, ko = torch.full_like(c.q, 7.0, memory_format=torch.contiguous_format), torch.full_like(c.k, 7.0, memory_format=torch.contiguous_format)
    dlm.qk_norm_rope(c.q, c.k, qo, ko, **c.how())
    check_heads(qo, *c.want(c.q, c.w[0]))
    check_heads(ko, *c.want(c.k, c.w[1]))
    if not norm and not rot:
        assert torch.equal(qo, c.q) and torch.equal(ko, c.k)


def test_layouts_one_tensor_and_in_place():
    c = Case(45, 6, 2, 128, 128, packed=False)
    qo, ko = torch.empty_like(c.q, memory_format=torch.contiguous_format), torch.empty(2, 45, 128, dtype=BF16, device=DEV).transpose(0, 1)
    dlm.qk_norm_rope(c.q, c.k, qo, ko, **c.how())
    check_heads(qo, *c.want(c.q, c.w[0]))
    check_heads(ko, *c.want(c.k, c.w[1]))
    only = torch.zeros_like(qo)
    dlm.qk_norm_rope(c.q, None, only, None, **c.how())
    assert torch.equal(only, qo)
    only = torch.zeros_like(ko)
    dlm.qk_norm_rope(None, c.k, None, only, **c.how())
    assert torch.equal(only, ko)
    one = c.q[:1].expand(45, 6, 128)                 # one token's heads, broadcast
    dlm.qk_norm_rope(one, None, only := torch.zeros_like(qo), None, **c.how())
    check_heads(only, *c.want(one, c.w[0]))
    dlm.qk_norm_rope(c.q, c.k, c.q, c.k, **c.how())
    assert torch.equal(c.q, qo) and torch.equal(c.k, ko)


def test_positions_outside_the_table_and_what_is_not_finite():
    c = Case(6, 2, 1, 64, 32)
    c.pos[1], c.pos[3] = -1, 50
    c.q[4, 0, 5], c.q[5, 1, 0] = float("nan"), float("inf")
    qo, ko = torch.zeros_like(c.q, memory_format=torch.contiguous_format), torch.zeros_like(c.k, memory_format=torch.contiguous_format)
    dlm.qk_norm_rope(c.q, c.k, qo, ko, **c.how())
    bad = torch.zeros(6, dtype=torch.bool, device=DEV)
    bad[[1, 3]] = True
    assert qo[bad][..., :32].isnan().all() and qo[bad][..., 32:].isfinite().all()
    assert ko[~bad].isfinite().all()
    assert qo[4, 0].isnan().all() and qo[4, 1].isfinite().all()                     # of that head, and of no other
    assert qo[5, 1, 0].isnan() and qo[5, 0].isfinite().all()


def test_zero_heads_and_far_positions():
    """A head of zeros stays zero; position 200 000 has the angle of the table."""
    c = Case(4, 2, 2, 128, 128, n_pos=200001)
    c.pos[0] = 200000
    c.q[2] = 0
    qo, ko = torch.empty_like(c.q, memory_format=torch.contiguous_format), torch.empty_like(c.k, memory_format=torch.contiguous_format)
    dlm.qk_norm_rope(c.q, c.k, qo, ko, **c.how())
    check_heads(qo, *c.want(c.q, c.w[0]))
    assert (qo[2] == 0).all()


@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("style", [dlm.ROPE_HALVES, dlm.ROPE_PAIRS])
@pytest.mark.parametrize("T,Hq,Hkv,d,rot", SHAPES + [(4099, 32, 2, 64, 64)])
def test_backward(T, Hq, Hkv, d, rot, style, norm):
    c = Case(T, Hq, Hkv, d, rot, style, norm, seed=5)
    dy = [bf16(c.rng, *t.shape) for t in (c.q, c.k)]
    dx = [torch.full_like(t, 3.0, memory_format=torch.contiguous_format) for t in (c.q, c.k)]
    dw = [torch.full((d,), 5.0, device=DEV) for _ in range(2)]
    ws = torch.empty(dlm.qk_norm_rope_bwd_workspace_bytes(T, Hq, Hkv, d), dtype=torch.uint8, device=DEV)
    given = dict(q=c.q, k=c.k, d_q_weight=dw[0], d_k_weight=dw[1], workspace=ws) if norm else {}
    dlm.qk_norm_rope_bwd(dy[0], dy[1], dx[0], dx[1], **given, **c.how())
    again = [t.clone() for t in dx + dw]
    for t, g, x, w, gw in zip((c.q, c.k), dy, dx, c.w, dw):
        check_gradient(c, t, g, x, w, gw if norm else None)
    dlm.qk_norm_rope_bwd(dy[0], dy[1], dx[0], dx[1], **given, **c.how())
    assert all(torch.equal(a, b) for a, b in zip(again, dx + dw))


def check_gradient(c, t, dy, got, w, got_w):
    x, g, pos = wide(t), wide(dy), c.pos.cpu().numpy()
    ww = None if w is None else wide(w)
    want, want_w = heads.head_map_grad(g, x, ww, EPS, c.table(), pos, c.style)
    size = np.abs(g)
    if c.rope is not None:
        i, j = heads._pairs(c.d, c.rope.shape[1], c.style)
        size[..., i] = size[..., j] = np.hypot(g[..., i], g[..., j])
    add = size
    if w is not None:
        r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + EPS)
        n, add = np.abs(x) * r, size * np.abs(ww)
        add = r * (add + n * (add * n).mean(-1, keepdims=True))
    err = np.abs(wide(got) - want)
    assert (err <= H * np.abs(want) * (1 + H) + 400 * U * add * (1 + H) + 2.0 ** -133).all()
    if got_w is not None:
        assert (np.abs(wide(got_w) - want_w) <= 400 * U * (size * n).sum((0, 1))).all()


def test_backward_of_part_of_it():
    """One tensor; no weight's gradient wanted; a broadcast input; in place of the upstream gradient; no tokens."""
    c = Case(77, 6, 2, 128, 128)
    dy, ws = bf16(c.rng, 77, 6, 128), torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
    dx, dw = torch.empty_like(dy), torch.full((128,), 9.0, device=DEV)
    dlm.qk_norm_rope_bwd(dy, None, dx, None, q=c.q, d_q_weight=dw, workspace=ws, **c.how())
    check_gradient(c, c.q, dy, dx, c.w[0], dw)
    alone = torch.empty_like(dy)
    dlm.qk_norm_rope_bwd(dy, None, alone, None, q=c.q, **c.how())
    assert torch.equal(alone, dx)
    one = c.q[:1].expand(77, 6, 128)
    dlm.qk_norm_rope_bwd(dy, None, alone, None, q=one, d_q_weight=dw, workspace=ws, **c.how())
    check_gradient(c, one, dy, alone, c.w[0], dw)
    dlm.qk_norm_rope_bwd(dy, None, dy, None, q=c.q, **c.how())
    assert torch.equal(dy, dx)
    c.pos = c.pos[:0]
    dlm.qk_norm_rope_bwd(dy[:0], None, dx[:0], None, q=c.q[:0], d_q_weight=dw, workspace=ws, **c.how())
    assert (dw == 0).all()


# ---- append ---------------------------------------------------------------------------------------------------------
def pool(rng, n, H, page, d, e4m3, token_major=False):
    """Two caches of the same strides, with other rows than the heads have."""
    got = []
    for _ in range(2):
        x = bf16(rng, n, page, H, d) * 8.0 if token_major else bf16(rng, n, H, page, d) * 8.0
        x = x.to(torch.float8_e4m3fn) if e4m3 else x
        got.append(x.transpose(1, 2) if token_major else x)
    return got


APPEND = [(1, 1, 1, 64, 64, 16), (1, 32, 8, 128, 128, 64), (7, 14, 2, 64, 32, 16), (64, 32, 8, 128, 128, 32), (193, 28, 4, 128, 0, 128), (515, 4, 4, 64, 64, 256)]


@pytest.mark.parametrize("token_major", [False, True])
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("T,Hq,Hkv,d,rot,page", APPEND)
def test_append(T, Hq, Hkv, d, rot, page, e4m3, token_major):
    c = Case(T, Hq, Hkv, d, rot, style=T % 2, norm=T != 64, seed=9)
    n = T // page + 4
    ck, cv = pool(c.rng, n, Hkv, page, d, e4m3, token_major)
    before = wide(ck), wide(cv)
    slots = c.rng.permutation(n * page)[:T].astype(np.int32)
    lost = c.rng.random(T) < 0.2
    slots[lost] = np.where(c.rng.random(lost.sum()) < 0.5, -1, n * page + 3)
    ks, vs = (torch.from_numpy((0.01 + 0.02 * c.rng.random(Hkv)).astype(np.float32)).to(DEV) if e4m3 else None for _ in range(2))
    qo = torch.full_like(c.q, 3.0, memory_format=torch.contiguous_format)
    dlm.paged_append(c.k, c.v, ck, cv, torch.from_numpy(slots).to(DEV), q=c.q, q_out=qo, k_scale=ks, v_scale=vs, **c.how())
    check_heads(qo, *c.want(c.q, c.w[0]))
    keys, size = c.want(c.k, c.w[1])
    for got, old, y, sz, scale in ((wide(ck), before[0], keys, size, ks), (wide(cv), before[1], wide(c.v), np.zeros(c.v.shape), vs)):
        touched = np.zeros((n, page), dtype=bool)
        for t in range(T):
            if lost[t]:
                continue
            p, row = divmod(int(slots[t]), page)
            touched[p, row] = True
            if e4m3:
                s = wide(scale)[:, None]
                x = y[t] / s
                # the nearest value, but for the error that the quotient carries: the heads' and three roundings of its own
                slack = 128 * U * sz[t] / s + 4 * U * np.abs(x)
                assert (np.abs(got[p, :, row] - np.clip(x, -448, 448)) <= heads.e4m3_distance(np.clip(x, -448, 448)) + 2 * slack).all()
            else:
                assert (np.abs(got[p, :, row] - y[t]) <= H * np.abs(y[t]) * (1 + H) + 128 * U * sz[t] * (1 + H) + 2.0 ** -133).all()
        assert np.array_equal(got.transpose(0, 2, 1, 3)[~touched], old.transpose(0, 2, 1, 3)[~touched])


def test_append_of_what_8_bits_do_not_hold():
    """Beyond the largest, infinities, NaN, and every border between two values with its ties."""
    vals = np.sort(heads.e4m3_values()[:127])
    ties = (vals[1:] + vals[:-1]) / 2
    x = np.concatenate([vals, -ties, ties, [449, 1e6, np.inf, -np.inf, np.nan]])
    assert len(x) == 384
    v = torch.from_numpy(x.astype(np.float32)).to(BF16).to(DEV)
    exact = wide(v)
    v = v.view(3, 1, 128)
    ck, cv = (torch.zeros((1, 1, 16, 128), dtype=torch.float8_e4m3fn, device=DEV) for _ in range(2))
    dlm.paged_append(torch.zeros_like(v), v, ck, cv, torch.tensor([0, 1, 2], dtype=I32, device=DEV))
    got = wide(cv)[0, 0, :3].reshape(-1)
    assert np.array_equal(np.isnan(got), np.isnan(exact))
    fine = ~np.isnan(exact)
    y = np.clip(exact[fine], -448, 448)
    want = torch.from_numpy(y.astype(np.float32)).to(torch.float8_e4m3fn).double().numpy()         # nearest, ties to even
    assert np.array_equal(got[fine], want)


def test_append_without_queries_tokens_or_room():
    c = Case(5, 4, 2, 128, 128)
    ck, cv = pool(c.rng, 2, 2, 16, 128, False)
    kept = ck.clone(), cv.clone()
    none = torch.full((5,), -1, dtype=I32, device=DEV)
    dlm.paged_append(c.k, c.v, ck, cv, none, **c.how())
    dlm.paged_append(c.k, c.v, ck[:0], cv[:0], none + 1, **c.how())                    # a cache of no pages
    assert torch.equal(ck, kept[0]) and torch.equal(cv, kept[1])
    c.pos = c.pos[:0]
    dlm.paged_append(c.k[:0], c.v[:0], ck, cv, none[:0], **c.how())
    assert torch.equal(ck, kept[0])


def test_rows_past_32_bits_of_offset():
    """A page 2^31 entries behind the first, and a token as far."""
    d, page, H = 64, 16, 1
    flat = torch.zeros((1 << 31) + 2 * page * d + d, dtype=BF16, device=DEV)
    ck = flat.as_strided((2, H, page, d), (1 << 31, page * d, d, 1))
    cv = flat.as_strided((2, H, page, d), (1 << 31, page * d, d, 1), page * d)
    x = flat.as_strided((2, 1, d), (1 << 31, d, 1), 2 * page * d)
    x[0], x[1] = 1.0, 2.0
    dlm.paged_append(x, x, ck, cv, torch.tensor([3, 21], dtype=I32, device=DEV))
    assert (ck[0, 0, 3] == 1).all() and (ck[1, 0, 5] == 2).all() and (cv[1, 0, 5] == 2).all() and (cv[0, 0, 3] == 1).all()
    assert int((flat != 0).sum()) == 6 * d


def refused(match, fn, *args, **kw):
    with pytest.raises(ValueError, match=match):
        fn(*args, **kw)


def test_binding_refuses_tensors_that_do_not_fit():
    x, w = torch.zeros((4, 2, 64), dtype=BF16, device=DEV), torch.zeros(64, dtype=BF16, device=DEV)
    i4, table = torch.zeros(4, dtype=I32, device=DEV), torch.zeros((8, 64), device=DEV)
    refused("goes with", dlm.qk_norm_rope, x, x, x, None)
    refused("axis 0, expected 4", dlm.qk_norm_rope, x, x[:3], x, x[:3])
    refused("dtype Float", dlm.qk_norm_rope, x.float(), None, x, None)
    refused("innermost", dlm.qk_norm_rope, x.transpose(1, 2), None, x.transpose(1, 2), None)
    refused("q_weight: size 64", dlm.qk_norm_rope, x[..., :32], None, x[..., :32], None, q_weight=w)
    refused("needs positions", dlm.qk_norm_rope, x, None, x, None, rope=table)
    refused("positions: size 4", dlm.qk_norm_rope, x[:3], None, x[:3], None, rope=table, positions=i4)
    refused("rope: must be contiguous", dlm.qk_norm_rope, x, None, x, None, rope=table[:, :32], positions=i4)
    refused("GPU", dlm.qk_norm_rope, x, None, x, None, q_weight=w.cpu())
    refused("a tensor", dlm.qk_norm_rope, x, None, [1], None)
    refused("goes with", dlm.qk_norm_rope_bwd, x, None, None, None)
    pages = torch.zeros((2, 2, 16, 64), dtype=BF16, device=DEV)
    refused("expected 2", dlm.paged_append, x, x, pages[:, :1], pages[:, :1], i4)
    refused("strides", dlm.paged_append, x, x, pages, pages.transpose(1, 2).contiguous().transpose(1, 2), i4)
    refused("slots", dlm.paged_append, x, x, pages, pages, None)
    refused("v: is needed", dlm.paged_append, x, None, pages, pages, i4)
    refused("dtype", dlm.paged_append, x, x, pages.half(), pages.half(), i4)
    q, tab, two = torch.zeros((2, 1, 4, 64), dtype=BF16, device=DEV), torch.zeros((2, 3), dtype=I32, device=DEV), torch.zeros(2, dtype=I32, device=DEV)
    refused("exceeds the 48", dlm.paged_attn, q, q.clone(), pages, pages, tab, two, max_kv_len=49)
    refused("block_table", dlm.paged_attn, q, q.clone(), pages, pages, tab[:1], two)
    refused("kv_len", dlm.paged_attn, q, q.clone(), pages, pages, tab, two.long())
    refused("lse", dlm.paged_attn, q, q.clone(), pages, pages, tab, two, lse=torch.zeros((2, 1, 4), device=DEV))
    with pytest.raises(dlm.DlmError, match="power of two") as e:
        dlm.paged_attn(q, q.clone(), pages[:, :, :15], pages[:, :, :15], tab, two)
    assert e.value.code == dlm.DLM_ERR_INVALID_ARG
