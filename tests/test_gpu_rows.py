"""Embedding and the norms between layers, forward and backward, against the 64-bit definitions (GPU).

Bounds, u = 2^-24 (half a step of fp32), h = 2^-8 (half a step of bf16).
Embedding: one product, then the rounding of the output.  Its gradient: a sum that goes through a chunk (64 rows at most), 16 chunks and groups of 16
chunks, at least 128 rows each: an entry passes 160 + n / 128 additions at most, one product by the scale, one addition to what was there.
Norm: sums over at most 32 entries a thread, 6 steps in a wavefront and 16 wavefronts: 56 u of what is added up.  The factor r is a root
of such a sum: 28 u, and 8 for its own operations.  The mean of a layer norm has 56 u of the mean of |x|, of which the second mean
leaves 56 u again: rows d are off by 2 u |d| + 60 u rms(d) + (60 u)^2 mean|x|.  So y / w is off by at most (64 + 44 |n|) u, plus r (60 u)^2 mean|x|.
Gradient of the norm: the same errors of n and r and sums of D products of two such numbers: 256 u of everything that is added up.  Columns: T rows in
teams, 64 or fewer rows each at these sizes, 32 teams, then workgroups in stretches: 600 u of what is added up."""
import numpy as np
import pytest
import torch

from oracle import rows
from paper_2604_04215_amd import binding as dlm
from gpu_util import DEV, GuardedWorkspace

pytestmark = pytest.mark.gpu
U, H = 2.0 ** -24, 2.0 ** -8
BF16, F32, I32, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


def wide(t):
    return t.detach().double().cpu().numpy()


def rnd(rng, *shape, dtype=BF16, std=1.0):
    return torch.from_numpy((rng.standard_normal(shape) * std).astype(np.float32)).to(dtype).to(DEV)


def within(got, want, inner):
    """One rounding to the output's type behind an error of `inner`."""
    step = H if got.dtype == BF16 else U
    err = np.abs(wide(got) - want)
    bound = step * np.abs(want) + inner * (1 + step) + 2.0 ** -133
    assert (err <= bound).all(), (err / bound).max()


def strided(t, gap):
    """The same rows further apart, garbage in between."""
    wide_ = torch.full((t.shape[0], t.shape[1] + gap), float("nan"), dtype=t.dtype, device=DEV)
    view = wide_[:, :t.shape[1]]
    view.copy_(t)
    return view


# ---- embedding ----------------------------------------------------------------------------------------------
def tokens_of(rng, T, V, masked=0.4, bad=0.1):
    t = rng.integers(0, V, T)
    t[rng.random(T) < masked] = V - 1
    t[rng.random(T) < bad] = -1
    t[rng.random(T) < bad / 2] = V
    if T > 2:
        t[1] = np.iinfo(np.int32).min
    return t.astype(np.int32)


@pytest.mark.parametrize("out_type", [BF16, F32])
@pytest.mark.parametrize("T,V,Dh,scale", [(1, 1, 8, 1.0), (1, 300, 64, 0.5), (5, 7, 72, -2.0), (33, 300, 200, 1.0), (100, 50, 512, 22.6), (17, 1000, 520, 1.0), (9, 20, 4096, 64.0),
                                          (3, 5, 8200, 1.0), (700, 2048, 256, 0.0)])
def test_embed(T, V, Dh, scale, out_type):
    rng = np.random.default_rng(T + V + Dh)
    tokens, table = tokens_of(rng, T, V), strided(rnd(rng, V, Dh), 24)
    out = strided(torch.full((T, Dh), 7.0, dtype=out_type, device=DEV), 8)
    dlm.embed(torch.from_numpy(tokens).to(DEV), table, out, scale=scale)
    want = rows.embed(tokens, wide(table), float(np.float32(scale)))
    within(out, want, U * np.abs(want))


def test_embed_of_a_table_with_infinities_and_padding():
    table = torch.zeros((3, 64), dtype=BF16, device=DEV)
    table[0, 3], table[1, 5] = float("inf"), float("nan")
    out = torch.full((4, 64), 7.0, dtype=F32, device=DEV)
    dlm.embed(torch.tensor([-1, 2, 1, 0], dtype=I32, device=DEV), table, out, scale=3.0)
    assert (out[:2] == 0).all() and out[2, 5].isnan() and out[2].isnan().sum() == 1 and out[3, 3].isinf() and out[3].isfinite().sum() == 63


def grad_of(tokens, d_out, d_table, **kw):
    ws = GuardedWorkspace(dlm.embed_bwd_workspace_bytes(len(tokens), *d_table.shape))
    dlm.embed_bwd(tokens, d_out, d_table, workspace=ws.ws, **kw)
    ws.check()


GRADS = [(1, 1, 8), (1, 300, 64), (2, 3, 264), (7, 7, 72), (16, 2, 512), (129, 5, 64), (333, 2048, 256), (1000, 40, 200), (2047, 300, 520), (2048, 9, 64), (2049, 9, 64), (513, 300, 64), (4100, 1 << 20, 8),
         (5000, 777, 1032), (70000, 1500, 64)]


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("in_type,out_type", [(BF16, F32), (F32, BF16), (BF16, BF16), (F32, F32)])
@pytest.mark.parametrize("T,V,Dh", GRADS)
def test_embed_gradient(T, V, Dh, in_type, out_type, accumulate):
    if T > 5000 and in_type != out_type:
        pytest.skip("large ones in two types")
    rng = np.random.default_rng(T + V + Dh)
    tokens, dy = tokens_of(rng, T, V), strided(rnd(rng, T, Dh, dtype=in_type), 16)
    table = strided(rnd(rng, V, Dh, dtype=out_type), 8)
    before = table.clone()
    grad_of(torch.from_numpy(tokens).to(DEV), dy, table, scale=1.7, accumulate=accumulate)
    d, size = rows.embed_grad(tokens, wide(dy), V, float(np.float32(1.7)))
    n = np.bincount(tokens[(tokens >= 0) & (tokens < V)], minlength=V)[:, None]
    if accumulate:
        d, size = d + wide(before), size + np.abs(wide(before))
        idle = torch.from_numpy(n[:, 0] == 0).to(DEV)
        assert torch.equal(table[idle], before[idle])           # neither read nor written
    within(table, d, (162 + n / 128) * U * size)


def test_embed_gradient_with_one_token_only_and_with_none():
    for T in (1, 127, 4096, 40000):
        dy, table = torch.ones((T, 64), dtype=BF16, device=DEV), torch.full((5, 64), 3.0, dtype=F32, device=DEV)
        grad_of(torch.full((T,), 2, dtype=I32, device=DEV), dy, table)
        assert (table[2] == T).all() and (table[[0, 1, 3, 4]] == 0).all()
        dy.fill_(float("nan"))
        table.fill_(3.0)
        grad_of(torch.full((T,), -1, dtype=I32, device=DEV), dy, table, accumulate=True)
        assert (table == 3).all()
        grad_of(torch.full((T,), 5, dtype=I32, device=DEV), dy, table)
        assert (table == 0).all()


def test_embed_gradient_of_no_tokens():
    table, none = torch.full((70, 72), 3.0, dtype=BF16, device=DEV), torch.zeros((0, 72), dtype=BF16, device=DEV)
    dlm.embed_bwd(torch.zeros(0, dtype=I32, device=DEV), none, table, accumulate=True)
    assert (table == 3).all()
    dlm.embed_bwd(torch.zeros(0, dtype=I32, device=DEV), none, table)
    assert (table == 0).all()


@pytest.mark.parametrize("kind", ["ascending", "descending", "runs", "two"])
def test_embed_gradient_of_orders_that_cut_chunks_everywhere(kind):
    """Small whole numbers: every sum is exact, so every row has to be there once."""
    T, Dh = 9001, 72
    at = np.arange(T)
    tokens = {"ascending": at, "descending": at[::-1], "runs": at // 37 * 5 % 400, "two": (at % 2) * 8999}[kind].astype(np.int32)
    dy = torch.from_numpy((at[:, None] * 7 + np.arange(Dh)) % 13 - 6).to(BF16).to(DEV)
    table = torch.full((T, Dh), float("nan"), dtype=F32, device=DEV)
    grad_of(torch.from_numpy(tokens.copy()).to(DEV), dy, table)
    assert np.array_equal(wide(table), rows.embed_grad(tokens, wide(dy), T, 1.0)[0])


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("kind", ["ascending", "descending", "mixed", "one run lacks what fills the others", "half of one", "none"])
@pytest.mark.parametrize("T", [2305, 8193, 70000, 140001])
def test_embed_gradient_merges_runs_of_any_order(T, kind, accumulate):
    """Exact again, over one and two levels of merging; tokens that one stretch of the list lacks and the others are full of."""
    V, Dh, rng = 70000, 8, np.random.default_rng(T)
    at = np.arange(T)
    few = np.where(at < 2048, at % 2 * 100, 50)
    tokens = {"ascending": at * V // T, "descending": (T - 1 - at) * V // T, "mixed": rng.integers(-5, V + 5, T), "one run lacks what fills the others": few,
              "half of one": np.where(rng.random(T) < 0.5, V - 1, rng.integers(0, 300, T)), "none": np.full(T, -1)}[kind].astype(np.int32)
    dy = torch.from_numpy((at[:, None] * 7 + np.arange(Dh)) % 13 - 6).to(BF16).to(DEV)
    table = torch.full((V, Dh), 3.0, dtype=F32, device=DEV)
    grad_of(torch.from_numpy(tokens).to(DEV), dy, table, accumulate=accumulate)
    want = np.zeros((V, Dh))
    live = (tokens >= 0) & (tokens < V)
    np.add.at(want, tokens[live], wide(dy)[live])
    assert np.array_equal(wide(table), want + (3 if accumulate else 0))


def test_embed_gradient_is_the_same_every_time_and_over_two_levels_of_merging():
    T, V = 140001, 90000                                        # 35 runs: more than are merged at once
    rng = np.random.default_rng(3)
    tokens, dy = torch.from_numpy(tokens_of(rng, T, V)).to(DEV), rnd(rng, T, 64)
    a, b = (torch.zeros((V, 64), dtype=F32, device=DEV) for _ in range(2))
    grad_of(tokens, dy, a)
    for _ in range(3):
        b.fill_(7.0)
        grad_of(tokens, dy, b)
        assert torch.equal(a, b)


def test_rows_beyond_32_bits():
    """A table and an output of which the last rows lie behind 2^31 entries."""
    stride, V = 1 << 22, 600
    big = torch.empty(V * stride, dtype=BF16, device=DEV)
    table = big.view(V, stride)[:, :64]
    table.copy_((torch.arange(V, device=DEV) % 128)[:, None].expand(V, 64))
    tokens = torch.tensor([0, 599, 513, 599, 512, -1], dtype=I32, device=DEV)
    out = torch.zeros((6, 64), dtype=F32, device=DEV)
    dlm.embed(tokens, table, out)
    assert out[:, 0].tolist() == [0, 87, 1, 87, 0, 0]
    grad_of(tokens, torch.ones_like(out), table, accumulate=True)
    assert table[[599, 513, 512, 0, 1], 63].tolist() == [89, 2, 1, 1, 1]
    dlm.row_norm(table, out2 := torch.zeros((V, 64), dtype=BF16, device=DEV))
    assert torch.equal(out2, (table > 0).to(BF16))
    dlm.row_norm_bwd(torch.ones_like(out2), table, table)
    # equal entries: r (g - mean(g)) = 0 but for eps; rows of zeros: r g = 1 / sqrt(1e-6)
    assert table[out2 == 1].abs().max() < 1e-2 and (table[out2 == 0] == 1000).all()


# ---- norms --------------------------------------------------------------------------------------------------
NORMS = [(1, 8), (1, 64), (7, 64), (33, 72), (5, 128), (300, 136), (9, 256), (2, 264), (13, 512), (3, 520), (2100, 896), (4, 1024), (2050, 1032), (5, 2048), (2051, 2056),
         (3, 3584), (2049, 4096), (2, 4104), (2070, 4104), (3, 8192), (2, 8200), (2053, 8200), (2, 16384)]


class Norm:
    def __init__(self, T, D, layer, dtype, affine=2, seed=0, mean=0.0):
        rng = np.random.default_rng(100 * T + D + seed)
        self.T, self.D, self.layer, self.eps = T, D, layer, 1e-5
        self.x = strided(rnd(rng, T, D, dtype=dtype) + mean, 16)
        self.res, self.ds = strided(rnd(rng, T, D, dtype=dtype), 8), strided(rnd(rng, T, D, dtype=dtype), 24)
        self.dy = strided(rnd(rng, T, D), 32)
        self.w = (1 + 0.3 * rnd(rng, D).float()).to(BF16) if affine else None
        self.b = rnd(rng, D) if affine == 2 else None
        self.kind = dlm.NORM_LAYER if layer else dlm.NORM_RMS

    def wb(self):
        return [None if t is None else wide(t) for t in (self.w, self.b)]

    def check_forward(self, out, x):
        w, b = self.wb()
        n, r = rows.normalise(x, self.layer, float(np.float32(self.eps)))
        inner = ((64 + 44 * np.abs(n)) * U + r * (60 * U) ** 2 * np.abs(x).mean(-1, keepdims=True)) * (1 if w is None else np.abs(w))
        want = rows.row_norm(x, self.layer, float(np.float32(self.eps)), w, b)
        within(out, want, inner + 2 * U * np.abs(want))

    def check_backward(self, dx, dw, db, x, ds):
        w, _ = self.wb()
        eps, dy = float(np.float32(self.eps)), wide(self.dy)
        n, r = rows.normalise(x, self.layer, eps)
        g = dy if w is None else dy * w
        mean = lambda v: np.abs(v).mean(-1, keepdims=True)
        want = rows.row_norm_grad(dy, x, self.layer, eps, w, ds)
        inner = 256 * U * r * (np.abs(g) + mean(g) + (np.abs(n) + 1) * (mean(g * n) + mean(g)))
        within(dx, want[0], inner + (0 if ds is None else 2 * U * np.abs(ds)))
        for got, d, size in ((dw, want[1], (np.abs(dy) * (np.abs(n) + 1)).sum(0)), (db, want[2], np.abs(dy).sum(0))):
            if got is not None:
                assert (np.abs(wide(got) - d) <= 600 * U * size + 2.0 ** -133).all(), (np.abs(wide(got) - d) / size).max() / U

    def backward(self, d_x, d_sum, sums=True):
        d_w, d_b = (torch.full((self.D,), 7.0, dtype=F32, device=DEV) if sums else None for _ in range(2))
        ws = GuardedWorkspace(dlm.row_norm_bwd_workspace_bytes(self.T, self.D))
        dlm.row_norm_bwd(self.dy, self.x, d_x, kind=self.kind, weight=self.w, eps=self.eps, d_sum=d_sum, d_weight=d_w, d_bias=d_b, workspace=ws.ws if sums else None)
        ws.check()
        return d_w, d_b


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("T,D", NORMS)
def test_norm(T, D, layer, dtype):
    c = Norm(T, D, layer, dtype, affine=(T + D) % 3)
    out = strided(torch.full((T, D), 7.0, dtype=BF16, device=DEV), 8)
    dlm.row_norm(c.x, out, kind=c.kind, weight=c.w, bias=c.b, eps=c.eps)
    c.check_forward(out, wide(c.x))
    total, again = strided(torch.full((T, D), 7.0, dtype=dtype, device=DEV), 8), torch.zeros_like(out)
    dlm.row_norm(c.x, out, kind=c.kind, weight=c.w, bias=c.b, eps=c.eps, residual=c.res, sum_out=total)
    assert torch.equal(total, (c.x.float() + c.res.float()).to(dtype))
    c.check_forward(out, wide(total))
    dlm.row_norm(c.x, again, kind=c.kind, weight=c.w, bias=c.b, eps=c.eps, residual=c.res)
    assert torch.equal(again, out)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("T,D", NORMS)
def test_norm_gradient(T, D, layer, dtype):
    c = Norm(T, D, layer, dtype, affine=(T + D) % 2)
    d_x = strided(torch.full((T, D), 7.0, dtype=dtype, device=DEV), 8)
    d_w, d_b = c.backward(d_x, c.ds)
    c.check_backward(d_x, d_w, d_b, wide(c.x), wide(c.ds))
    only = torch.zeros_like(d_x)
    c.backward(only, None, sums=False)
    c.check_backward(only, None, None, wide(c.x), None)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_norm_in_place_and_broadcast(dtype):
    c = Norm(37, 264, True, dtype)
    want, out, total = (torch.zeros((37, 264), dtype=t, device=DEV) for t in (BF16, BF16, dtype))
    how = dict(kind=c.kind, weight=c.w, bias=c.b, eps=c.eps)
    dlm.row_norm(c.x, want, residual=c.res, sum_out=total, **how)
    one = c.x[:1].expand(37, 264)
    dlm.row_norm(one, out, residual=c.res, **how)
    c.check_forward(out, wide((one.float() + c.res.float()).to(dtype)))
    res = c.res.clone()
    dlm.row_norm(c.x, out, residual=res, sum_out=res, **how)
    assert torch.equal(out, want) and torch.equal(res, total)
    x = c.x.clone()
    dlm.row_norm(x, out, residual=c.res, sum_out=x, **how)
    assert torch.equal(out, want) and torch.equal(x, total)
    d_x = torch.zeros_like(total)
    sums = c.backward(d_x, c.ds)
    for name in ("ds", "x") + (("dy",) if dtype == BF16 else ()):
        d = Norm(37, 264, True, dtype)
        buffer = getattr(d, name)
        again = d.backward(buffer, d.ds)
        assert torch.equal(buffer, d_x) and all(torch.equal(a, b) for a, b in zip(sums, again))
    if dtype == BF16:
        x = c.x.clone()
        dlm.row_norm(x, x, **how)
        dlm.row_norm(c.x, want, **how)
        assert torch.equal(x, want)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_layer_norm_of_rows_far_from_zero(dtype):
    """All equal, or far from zero with little deviation: the mean's own rounding must not show."""
    for T, D in ((3, 72), (2, 1032), (2100, 1032), (2, 16384)):
        c = Norm(T, D, True, dtype, affine=0)
        c.x.fill_(1000.1)
        out = torch.full((T, D), 7.0, dtype=BF16, device=DEV)
        dlm.row_norm(c.x, out, kind=c.kind, eps=1e-12)
        assert (out.abs() <= 1000.1 * (60 * U) ** 2 * 1e6 * 1.1 + 1e-30).all()
        c = Norm(T, D, True, dtype, affine=2, mean=300.0)
        dlm.row_norm(c.x, out, kind=c.kind, weight=c.w, bias=c.b, eps=c.eps)
        c.check_forward(out, wide(c.x))
        d_x = torch.zeros_like(c.x, memory_format=torch.contiguous_format)
        c.check_backward(d_x, *c.backward(d_x, c.ds), wide(c.x), wide(c.ds))


@pytest.mark.parametrize("layer", [False, True])
def test_norm_of_zeros_and_what_is_not_finite(layer):
    T, D = 6, 520
    c = Norm(T, D, layer, BF16)
    c.x.copy_(torch.ones_like(c.x) * torch.arange(D, device=DEV))
    c.x[1].zero_()
    c.x[2, 3], c.x[3, 4], c.x[5, 0] = float("nan"), float("inf"), -float("inf")
    out = torch.zeros((T, D), dtype=BF16, device=DEV)
    dlm.row_norm(c.x, out, kind=c.kind, weight=c.w, bias=c.b, eps=c.eps)
    assert torch.equal(out[1], c.b) and out[2].isnan().all() and out[[0, 4]].isfinite().all()
    if layer:
        assert out[[3, 5]].isnan().all()
    else:
        assert out[3, 4].isnan() and out[5, 0].isnan()
    d_x = torch.zeros_like(c.x, memory_format=torch.contiguous_format)
    c.dy.copy_(torch.ones_like(c.dy))
    c.backward(d_x, None)
    assert d_x[[0, 1, 4]].isfinite().all() and d_x[2].isnan().all()


def test_norm_of_no_rows_and_of_more_than_a_launch_takes():
    d_w, d_b = (torch.full((64,), 7.0, dtype=F32, device=DEV) for _ in range(2))
    none = torch.zeros((0, 64), dtype=BF16, device=DEV)
    dlm.row_norm(none, none)
    dlm.row_norm_bwd(none, none, none, d_weight=d_w, d_bias=d_b)
    assert (d_w == 0).all() and (d_b == 0).all()
    T = (1 << 20) + 5
    x = torch.arange(T, device=DEV)[:, None].expand(T, 8).to(BF16) + 1
    out, total = torch.zeros((T, 8), dtype=BF16, device=DEV), torch.zeros((T, 8), dtype=BF16, device=DEV)
    dlm.row_norm(x, out, residual=x, sum_out=total)
    assert (out == 1).all() and torch.equal(total, x + x)


def test_on_another_stream_and_replayed_from_a_graph():
    rng = np.random.default_rng(5)
    T, V, D = 700, 90, 264
    c = Norm(T, D, True, F32)
    tokens, table = torch.from_numpy(tokens_of(rng, T, V)).to(DEV), rnd(rng, V, D)
    ws = torch.empty(max(dlm.embed_bwd_workspace_bytes(T, V, D), dlm.row_norm_bwd_workspace_bytes(T, D)), dtype=U8, device=DEV)

    def buffers():
        return dict(x=torch.zeros((T, D), dtype=F32, device=DEV), s=torch.zeros((T, D), dtype=F32, device=DEV), y=torch.zeros((T, D), dtype=BF16, device=DEV),
                    d_x=torch.zeros((T, D), dtype=F32, device=DEV), d_w=torch.zeros(D, dtype=F32, device=DEV), d_b=torch.zeros(D, dtype=F32, device=DEV),
                    d_table=torch.zeros((V, D), dtype=F32, device=DEV))

    def chain(b, **kw):
        dlm.embed(tokens, table, b["x"], scale=2.0, **kw)
        dlm.row_norm(b["x"], b["y"], kind=c.kind, weight=c.w, bias=c.b, residual=c.res, sum_out=b["s"], **kw)
        dlm.row_norm_bwd(c.dy, b["s"], b["d_x"], kind=c.kind, weight=c.w, d_sum=c.ds, d_weight=b["d_w"], d_bias=b["d_b"], workspace=ws, **kw)
        dlm.embed_bwd(tokens, b["d_x"], b["d_table"], scale=2.0, workspace=ws, **kw)

    eager, other, graphed = buffers(), buffers(), buffers()
    chain(eager)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    chain(other, stream=side)
    side.synchronize()
    assert all(torch.equal(eager[k], other[k]) for k in eager)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain(graphed)
    for k in range(4):
        tokens.copy_(torch.from_numpy(tokens_of(rng, T, V)).to(DEV))
        for v in graphed.values():
            v.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        chain(eager)
        torch.cuda.synchronize()
        assert all(torch.equal(eager[k], graphed[k]) for k in eager), k


@pytest.mark.parametrize("T", [100, 1500, 3000, 70000])
def test_whatever_the_workspaces_held(T):
    rng = np.random.default_rng(T)
    tokens, x, dy = torch.from_numpy(tokens_of(rng, T, 900)).to(DEV), rnd(rng, T, 72), rnd(rng, T, 72)
    outs = []
    for fill in (0, 0x3f, 0x80, 0xff):
        ws = [torch.full((n,), fill, dtype=U8, device=DEV) for n in (dlm.embed_bwd_workspace_bytes(T, 900, 72), dlm.row_norm_bwd_workspace_bytes(T, 72))]
        added, whole, d_x, d_w, d_b = torch.ones((900, 72), device=DEV), torch.ones((900, 72), device=DEV), torch.zeros_like(x), torch.zeros(72, device=DEV), torch.zeros(72, device=DEV)
        dlm.embed_bwd(tokens, dy, added, accumulate=True, workspace=ws[0])
        ws[0].fill_(fill)
        dlm.embed_bwd(tokens, dy, whole, workspace=ws[0])
        dlm.row_norm_bwd(dy, x, d_x, kind=dlm.NORM_LAYER, d_weight=d_w, d_bias=d_b, workspace=ws[1])
        outs.append((added, whole, d_x, d_w, d_b))
    assert all(torch.equal(a, b) for got in outs[1:] for a, b in zip(got, outs[0])) and all(t.isfinite().all() for t in outs[0])


def test_binding_checks():
    x, t = torch.zeros((4, 64), dtype=BF16, device=DEV), torch.zeros(4, dtype=I32, device=DEV)
    with pytest.raises(ValueError, match="dtype"):
        dlm.embed(t.long(), x, x)
    with pytest.raises(ValueError, match="size"):
        dlm.embed(t[:3], x, x)
    with pytest.raises(ValueError, match="dtype"):
        dlm.embed(t, x.float(), x)
    with pytest.raises(ValueError, match="dtype"):
        dlm.row_norm(x, x, residual=x.float())
    with pytest.raises(ValueError, match="contiguous"):
        dlm.row_norm(x, x.t())
    with pytest.raises(ValueError, match="size"):
        dlm.row_norm_bwd(x, x, x, weight=x[0, :32])
    with pytest.raises(ValueError, match="needed"):
        dlm.row_norm_bwd(x, x, None)
    with pytest.raises(dlm.DlmError) as e:
        dlm.embed_bwd(t, x, x.clone())
    assert e.value.code == dlm.DLM_ERR_WORKSPACE
    with pytest.raises(dlm.DlmError) as e:
        dlm.row_norm_bwd(x, x, x, d_weight=torch.zeros(64, dtype=F32, device=DEV))
    assert e.value.code == dlm.DLM_ERR_WORKSPACE
