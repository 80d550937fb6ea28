"""The LM head's gradient against the 64-bit definition (GPU).

Bounds, u = 2^-24 (half a step of fp32), h = 2^-8 (half a step of bf16).  A sum of K products on the matrix pipes: a product passes at most 16 additions in
its own instruction and K / 16 behind it; each may be off by 2 u (should it cut instead of round) of what is added up: s(K) = 2 u (16 + K / 16).
Logits are off by e = inv_t s(Dh) sum|h w| and 4 u (|z| + |lse|), probabilities by p (exp(e) - 1 + 8 u).  dz is then rounded: to three terms of bf16 for fp32
gradients, h^3 |dz|, to two up to 128 rows, h^2 |dz|, or to one fp16, 2^-11 |dz| or half its smallest step, 2^-25, of numbers up to 2^14: 2^-38 of the largest |dz| times
rows and columns of up to 2 in size.  A gradient is off by the sum of |its other operand| times that, by s(K) of what is added up (with up to 64 partial sums joined: 128 u more),
and by its own rounding."""
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


def s(K):
    return 2 * U * (16 + K / 16)


class Case:
    def __init__(self, M, Dh, V, *, seed=0, inv_t=1.0, forbid=-1, extra=0, rows_total=None, scatter=False, gap=0, wstd=None):
        rng = self.rng = np.random.default_rng(M * 7 + Dh + V + seed)
        self.M, self.Dh, self.V, self.inv_t, self.forbid, self.scatter = M, Dh, V, float(np.float32(inv_t)), forbid, scatter
        n = self.n = rows_total or M
        put = lambda x: torch.from_numpy(x.astype(np.float32)).to(BF16).to(DEV)

        def spread(x):                                   # the same rows further apart, garbage in between
            if not gap:
                return x
            t = torch.full((x.shape[0], x.shape[1] + gap), float("nan"), dtype=x.dtype, device=DEV)
            t[:, :x.shape[1]] = x
            return t[:, :x.shape[1]]

        self.hidden = spread(put(rng.standard_normal((n, Dh))))
        self.w = spread(put(rng.standard_normal((V, Dh)) * (Dh ** -0.25 if wstd is None else wstd)))
        self.idx = np.sort(rng.permutation(n)[:M]).astype(np.int32) if n > M else None
        h = self.h = wide(self.hidden)[self.idx] if self.idx is not None else wide(self.hidden)
        z = self.z = h @ wide(self.w).T * self.inv_t
        if forbid >= 0:
            z[:, forbid] = -np.inf
        top = z.max(1, keepdims=True)
        lse = (top + np.log(np.exp(z - top).sum(1, keepdims=True)))[:, 0]
        target = rng.integers(0, V, M)
        best = rng.random(M) < 0.3
        target[best] = z.argmax(1)[best]
        target[rng.random(M) < 0.1] = -1
        if M > 4:
            target[:4] = [V, forbid, 0, V - 1]
        self.lse, self.target = lse.astype(np.float32), target.astype(np.int32)
        g = rng.standard_normal(M).astype(np.float32)
        self.d_zt, self.d_lse = g, (-g + 0.1 * rng.standard_normal(M)).astype(np.float32)
        if M > 6:
            self.d_lse[5], self.lse[5] = 0.0, np.nan     # a row without this gradient may have any lse
            self.d_zt[6] = self.d_lse[6] = 0.0

    def arrays(self):
        """lse, target, d_ztarget, d_lse as the call wants them"""
        out = []
        for x in (self.lse, self.target, self.d_zt, self.d_lse):
            if self.scatter and self.idx is not None:
                y = np.full(self.n, 77, dtype=x.dtype)
                y[self.idx] = x
                x = y
            out.append(torch.from_numpy(x).to(DEV))
        return out

    def call(self, d_hidden, d_w, live=None, **kw):
        lse, target, d_zt, d_lse = self.arrays()
        how = dict(target=target, d_ztarget=d_zt, d_lse=d_lse, d_hidden=d_hidden, d_w=d_w, inv_temperature=self.inv_t, forbid_token=self.forbid, out_scatter=self.scatter)
        if self.idx is not None:
            how["row_idx"] = torch.from_numpy(self.idx).to(DEV)
        if live is not None:
            how["m_dev"] = torch.tensor([live], dtype=I32, device=DEV)
        how.update(kw)
        ws = GuardedWorkspace(dlm.lmhead_bwd_workspace_bytes(self.hidden, self.w, lse, **how))
        ws.ws.fill_(255)                                 # NaN, whatever the type
        dlm.lmhead_bwd(self.hidden, self.w, lse, workspace=ws.ws, **how)
        ws.check()

    def want(self, two_h, two_w, live=None, d_lse=True, d_zt=True):
        """(d_hidden, its bound, d_w, its bound) before the roundings of the results"""
        m = self.M if live is None else max(0, min(self.M, live))
        h, w = self.h[:m], wide(self.w)
        lse, a, c = (x[:m].astype(np.float64) for x in (self.lse, self.d_lse, self.d_zt))
        dz, dh, dw = rows.lmhead_grad(h, w, lse, a if d_lse else None, c if d_zt else None, self.target[:m], self.inv_t, self.forbid)
        e = self.inv_t * s(self.Dh) * (np.abs(h) @ np.abs(w).T) + 4 * U * (np.abs(np.where(np.isinf(self.z[:m]), 0, self.z[:m])) + np.abs(lse)[:, None])
        p = np.exp(np.where(np.isinf(self.z[:m]), -np.inf, self.z[:m]) - lse[:, None])
        off = np.where((a != 0)[:, None] & d_lse, np.abs(a)[:, None] * p * (np.expm1(e) + 8 * U) * self.inv_t, 0.0) + 4 * U * np.abs(dz) + 2.0 ** -126
        off = np.nan_to_num(off, nan=0.0)
        size, ah, aw = np.abs(dz), np.abs(h), np.abs(w)
        def part(wide_):
            if wide_:
                return off * (1 + H) + H ** 3 * size
            if self.M <= 128 or wide_any:
                return off * (1 + H) + H * H * size
            return off * (1 + H) + 2.0 ** -11 * size + 2.0 ** -36 * size.max(initial=0)

        wide_any = two_h or two_w
        bh = part(two_h) @ aw + (s(2 * self.V) + 128 * U) * ((size + off) @ aw) * 1.01
        bw = part(two_w).T @ ah + s(2 * m) * ((size + off).T @ ah) * 1.01
        return dh, bh, dw, bw


def within(got, want, bound):
    step = H if got.dtype == BF16 else U
    err = np.abs(wide(got) - want)
    ok = err <= step * np.abs(want) + bound * (1 + step) + 2.0 ** -126
    assert ok.all(), (np.argwhere(~ok)[:5], (err / (step * np.abs(want) + bound + 1e-30)).max())


def near(got, want, two):
    """In the norm.  The root mean square of many roundings of up to h is h / sqrt(3) = 0.58 h; what dz keeps, 11 bits or more, leaves the rest.  fp32: a logit's error is
    that of some 100 roundings of numbers of up to 8 or so, 2^-24 8 sqrt(100) / sqrt(3) = 3e-6."""
    if want.size and np.linalg.norm(want) > 0:
        rel = np.linalg.norm(wide(got) - want) / np.linalg.norm(want)
        assert rel <= (3e-6 if got.dtype == F32 else 0.6 * H if want.size > 1000 else H), rel


SHAPES = [(1, 64, 1), (256, 128, 400), (1, 64, 300), (2, 128, 65), (16, 256, 2048), (3, 64, 64), (64, 320, 777), (65, 192, 1000), (257, 64, 513), (300, 896, 1500), (130, 1024, 4099), (520, 576, 700),
          (33, 4096, 333)]


@pytest.mark.parametrize("types", [(BF16, BF16), (F32, F32), (BF16, F32), (F32, BF16)])
@pytest.mark.parametrize("M,Dh,V", SHAPES)
def test_gradient(M, Dh, V, types):
    c = Case(M, Dh, V, forbid=V - 1 if V > 1 and M % 2 == 0 else -1, inv_t=0.7 if M % 3 == 0 else 1.0, gap=16 if V % 2 else 0)
    d_h, d_w = (torch.full((n, Dh), float("nan"), dtype=t, device=DEV) for n, t in ((M, types[0]), (V, types[1])))
    c.call(d_h, d_w)
    dh, bh, dw, bw = c.want(types[0] == F32, types[1] == F32)
    within(d_h, dh, bh)
    within(d_w, dw, bw)
    near(d_h, dh, types[0] == F32)
    near(d_w, dw, types[1] == F32)


def check(c, types, live=None):
    d_h, d_w = (torch.full((n, c.Dh), float("nan"), dtype=t, device=DEV) for n, t in ((c.M, types[0]), (c.V, types[1])))
    c.call(d_h, d_w, live)
    dh, bh, dw, bw = c.want(types[0] == F32, types[1] == F32, live)
    within(d_h[:len(dh)], dh, bh)
    within(d_w, dw, bw)
    near(d_h[:len(dh)], dh, types[0] == F32)
    near(d_w, dw, types[1] == F32)
    assert d_h[len(dh):].isnan().all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,Dh,V", [(50, 64, 41000), (100, 128, 41003), (200, 64, 41000), (300, 64, 40961), (300, 320, 12000), (20, 704, 12000)])
def test_vocabularies_that_take_large_tiles(M, Dh, V, dtype):
    check(Case(M, Dh, V, forbid=V - 1), (dtype, dtype))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("live", [None, 60, 130])
@pytest.mark.parametrize("M,Dh,V", [(16, 64, 1000), (70, 448, 1601), (200, 128, 3000), (330, 320, 2003), (300, 128, 13000), (140, 64, 41000)])
def test_workgroups_that_take_one_tile_after_another(M, Dh, V, live, dtype):
    """Eight or sixteen workgroups for all tiles, so that each takes many: in one chunk and in several."""
    c = Case(M, Dh, V, forbid=3, gap=8 if V == 2003 else 0)
    for workgroups, columns in ((8, 0), (16, 1024)):
        dlm.set_option("lmhead_bwd_workgroups", workgroups)
        dlm.set_option("lmhead_bwd_columns", columns)
        try:
            check(c, (dtype, dtype), live)
        finally:
            dlm.set_option("lmhead_bwd_workgroups", 0)
            dlm.set_option("lmhead_bwd_columns", 0)


@pytest.mark.parametrize("scatter", [False, True])
@pytest.mark.parametrize("live", [None, 0, 1, 63, 64, 70, 1000, -5])
def test_rows_by_index_and_a_count_on_the_device(scatter, live):
    c = Case(100, 192, 777, rows_total=173, scatter=scatter, forbid=776, gap=8)
    d_h, d_w = torch.full((173, 200), 7.0, dtype=F32, device=DEV)[:, :192], torch.full((777, 200), 3.0, dtype=BF16, device=DEV)[:, :192]
    c.call(d_h, d_w, live)
    dh, bh, dw, bw = c.want(True, False, live)
    named = torch.from_numpy(c.idx[:len(dh)]).long().to(DEV)
    within(d_h[named], dh, bh)
    within(d_w, dw, bw)
    rest = torch.ones(173, dtype=torch.bool, device=DEV)
    rest[named] = False
    assert (d_h[rest] == 7).all()


@pytest.mark.parametrize("types", [(BF16, BF16), (F32, F32)])
@pytest.mark.parametrize("scatter", [False, True])
@pytest.mark.parametrize("M,named,live", [(70, 5, None), (300, 70, 290), (700, 1, None), (1000, 900, None), (5000, 3000, 4700)])
def test_rows_named_more_than_once_and_in_any_order(M, named, live, scatter, types):
    c = Case(M, 64, 200, rows_total=M + 1, scatter=False, forbid=3)
    c.scatter, c.n = scatter, named
    c.hidden, c.idx = c.hidden[:named].contiguous(), c.rng.integers(0, named, M).astype(np.int32)
    c.h = wide(c.hidden)[c.idx]
    c.z = c.h @ wide(c.w).T
    c.z[:, 3] = -np.inf
    c.lse = np.log(np.exp(c.z).sum(1)).astype(np.float32)
    if scatter:                                          # what belongs to a row is the same wherever it is named
        last = np.zeros(named, dtype=int)
        last[c.idx] = np.arange(M)
        c.lse, c.target, c.d_zt, c.d_lse = (x[last[c.idx]] for x in (c.lse, c.target, c.d_zt, c.d_lse))
    d_h, d_w = torch.full((named, 64), 7.0, dtype=types[0], device=DEV), torch.zeros((200, 64), dtype=types[1], device=DEV)
    c.call(d_h, d_w, live)
    again = torch.full_like(d_h, 7.0)
    c.call(again, d_w, live)
    assert torch.equal(d_h, again)
    dh, bh, dw, bw = c.want(types[0] == F32, types[1] == F32, live)
    want, bound, size = np.zeros((3, named, 64))
    idx = c.idx[:len(dh)]
    np.add.at(want, idx, dh)
    np.add.at(size, idx, np.abs(dh))
    np.add.at(bound, idx, bh)
    there = np.unique(idx)
    # up to M sums of a row are added one after the other: each addition half a step of what there is so far off
    within(d_h[torch.from_numpy(there).to(DEV)], want[there], bound[there] + U * np.bincount(idx, minlength=named).max() * size[there])
    within(d_w, dw, bw)
    assert (np.delete(wide(d_h), there, 0) == 7).all()


@pytest.mark.parametrize("M", [70, 300])
def test_in_the_place_of_the_hidden_rows(M):
    c = Case(M, 128, 300, rows_total=M + 30, forbid=3)
    d_h, d_w = torch.zeros((M + 30, 128), dtype=BF16, device=DEV), torch.zeros((300, 128), dtype=BF16, device=DEV)
    c.call(d_h, d_w)
    before, there = c.hidden.clone(), torch.from_numpy(c.idx).long().to(DEV)
    c.call(c.hidden, torch.zeros_like(d_w))
    assert torch.equal(c.hidden[there], d_h[there])
    before[there] = d_h[there]
    assert torch.equal(c.hidden, before)


def test_one_gradient_alone_and_one_cotangent_alone():
    c = Case(70, 128, 300, forbid=3)
    both_h, both_w = torch.zeros((70, 128), dtype=BF16, device=DEV), torch.zeros((300, 128), dtype=F32, device=DEV)
    c.call(both_h, both_w)
    d_h, d_w = torch.zeros_like(both_h), torch.zeros_like(both_w)
    c.call(d_h, None)
    c.call(None, d_w)
    dh, bh, dw, bw = c.want(False, True)
    for a, b, want, bound in ((d_h, both_h, dh, bh), (d_w, both_w, dw, bw)):
        within(a, want, bound)
        within(b, want, bound)
    for lse, zt in ((True, False), (False, True)):
        kw = {} if lse else dict(d_lse=None)
        kw.update({} if zt else dict(d_ztarget=None, target=None))
        c.call(d_h, d_w, **kw)
        dh, bh, dw, bw = c.want(False, True, d_lse=lse, d_zt=zt)
        within(d_h, dh, bh)
        within(d_w, dw, bw)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_accumulation_and_none_of_it(dtype):
    c = Case(90, 320, 1001)
    base = torch.from_numpy(c.rng.standard_normal((1001, 320)).astype(np.float32)).to(dtype).to(DEV)
    d_w = base.clone()
    c.call(None, d_w, accumulate=True)
    _, _, dw, bw = c.want(False, dtype == F32)
    within(d_w, dw + wide(base), bw + 2 * U * np.abs(wide(base)))
    d_w = base.clone()
    c.call(None, d_w, live=0, accumulate=True)
    assert torch.equal(d_w, base)
    c.call(None, d_w, live=0)
    assert (d_w == 0).all()
    none = torch.zeros((0, 320), dtype=BF16, device=DEV)
    f, i = torch.zeros(0, dtype=F32, device=DEV), torch.zeros(0, dtype=I32, device=DEV)
    ws = torch.empty(1 << 22, dtype=U8, device=DEV)
    d_w.copy_(base)
    dlm.lmhead_bwd(none, c.w, f, d_lse=f, d_ztarget=f, target=i, d_w=d_w, accumulate=True, workspace=ws)
    assert torch.equal(d_w, base)
    dlm.lmhead_bwd(none, c.w, f, d_lse=f, d_hidden=none, d_w=d_w, workspace=ws)
    assert (d_w == 0).all()


def test_rows_and_columns_of_very_different_size():
    """Many rows in 16 bits: dz is scaled by row and column.  Every row of d_hidden and of d_w has to be right by its own size."""
    c = Case(300, 192, 1000, forbid=999)
    rng = np.random.default_rng(8)
    power = rng.integers(-30, 1, 300)                        # of a row's gradient
    c.d_zt, c.d_lse = ((x * 2.0 ** power).astype(np.float32) for x in (c.d_zt, c.d_lse))
    put = lambda x: torch.from_numpy(x.astype(np.float32)).to(BF16).to(DEV)
    c.hidden = put(wide(c.hidden) * 2.0 ** rng.integers(-3, 4, (300, 1)))
    c.hidden[7].zero_()
    w = wide(c.w) * 2.0 ** rng.integers(-4, 2, (1000, 1))
    w[[3, 500]] = 0.0
    c.w, c.h = put(w), wide(c.hidden)
    c.z = c.h @ wide(c.w).T
    c.z[:, 999] = -np.inf
    c.lse = np.log(np.exp(c.z - 20).sum(1)).astype(np.float32) + np.float32(20)
    d_h, d_w = torch.zeros((300, 192), dtype=BF16, device=DEV), torch.zeros((1000, 192), dtype=BF16, device=DEV)
    c.call(d_h, d_w)
    dz, dh, dw = rows.lmhead_grad(c.h, wide(c.w), c.lse.astype(np.float64), c.d_lse.astype(np.float64), c.d_zt.astype(np.float64), c.target, 1.0, 999)
    # dz is 2^-11 off, or half the smallest step of what it is stored as: D = dz 2^(e + u + f - K), e and f the exponents of the largest entries of its
    # rows of hidden and W, K = max(e + c) + max(f) - 13, c the exponent of |d_lse| + |d_ztarget|, u = min(max(e + c) - e - c, 20)
    exponent = lambda x: np.floor(np.log2(np.where(x > 0, x, 1)))
    top_h, top_w, g = np.abs(c.h).max(1), np.abs(wide(c.w)).max(1), np.abs(c.d_lse.astype(np.float64)) + np.abs(c.d_zt)
    e, f, k = exponent(top_h), exponent(top_w), exponent(g)
    most, f = (e + k)[(top_h > 0) & (g > 0)].max(), np.where(top_w > 0, f, f[top_w > 0].max())
    u = np.where((top_h > 0) & (g > 0), np.minimum(most - e - k, 20), 0)
    least = 2.0 ** (-25 + (most + f.max() - 13) - (e + u)[:, None] - f)
    off = np.expm1(s(192) * (np.abs(c.h) @ np.abs(wide(c.w)).T) + 8 * U * (np.abs(c.lse)[:, None] + 50))
    extra = np.abs(c.d_lse)[:, None] * np.exp(np.where(np.isinf(c.z), -np.inf, c.z) - c.lse[:, None]) * off
    size = np.abs(dz) * (2.0 ** -11 + off) + extra + least
    within(d_h, dh, (size + s(1000) * np.abs(dz)) @ np.abs(wide(c.w)) * 1.01)
    # (entries of hidden rows that u brings down below the smallest normal fp16 are half of its smallest step off, 2^-19 of the row's largest)
    within(d_w, dw, ((size + s(300) * np.abs(dz)).T @ np.abs(c.h) + np.abs(dz).T @ (2.0 ** -18 * top_h)[:, None]) * 1.01)


@pytest.mark.parametrize("M,zeros,size", [(200, 200, 1.0), (300, 300, 2.0 ** 30), (200, 1, 2.0 ** -30), (260, 259, 2.0 ** 20)])
def test_hidden_rows_of_zeros(M, zeros, size):
    """Their gradient is not zero, and no other row's size is theirs."""
    c = Case(M, 128, 333, forbid=7)
    c.d_zt, c.d_lse = (np.nan_to_num(x) * np.float32(1000.0) for x in (c.d_zt, c.d_lse))
    c.lse = np.nan_to_num(c.lse)
    hidden = wide(c.hidden) * size
    hidden[M - zeros:] = 0.0
    w = wide(c.w) / max(size, 1.0)                       # logits of ordinary size
    c.hidden, c.w = (torch.from_numpy(x.astype(np.float32)).to(BF16).to(DEV) for x in (hidden, w))
    c.h = wide(c.hidden)
    c.z = c.h @ wide(c.w).T
    c.z[:, 7] = -np.inf
    c.lse = np.log(np.exp(c.z).sum(1)).astype(np.float32)
    d_h, d_w = (torch.full((n, 128), float("nan"), dtype=BF16, device=DEV) for n in (M, 333))
    c.call(d_h, d_w)
    dh, bh, dw, bw = c.want(False, False)
    # dz of a row is 2^-11 off, or half the smallest step of what it is stored as: 2^-38 of the row's largest times W's sizes' spread, at most 2^10 here; the
    # columns' largest entries differ by less
    within(d_h, dh, bh + 2.0 ** -28 * np.abs(dh).max(1, keepdims=True))
    within(d_w, dw, bw + 2.0 ** -28 * np.abs(dw).max())
    near(d_h, dh, False)


@pytest.mark.parametrize("M", [100, 200])
@pytest.mark.parametrize("rows_of", ["half", "but one", "all"])
def test_small_rows_of_w(M, rows_of):
    """Their own gradient is not small: it is of dz and the hidden rows alone."""
    c = Case(M, 128, 1000, forbid=999)
    small = np.ones(1000)
    small[::2 if rows_of == "half" else 1] = 2.0 ** -24
    if rows_of == "but one":
        small[500] = 1.0
    c.w = torch.from_numpy((wide(c.w) * small[:, None]).astype(np.float32)).to(BF16).to(DEV)
    c.z = c.h @ wide(c.w).T
    c.z[:, 999] = -np.inf
    c.lse = np.log(np.exp(c.z).sum(1)).astype(np.float32)
    d_h, d_w = (torch.full((n, 128), float("nan"), dtype=BF16, device=DEV) for n in (M, 1000))
    c.call(d_h, d_w)
    dh, bh, dw, bw = c.want(False, False)
    # dz is at most half the smallest step off, 2^-39 of the largest number, which is at most 2^9 times the largest product of a gradient and its row
    within(d_w, dw, bw)
    near(d_w, dw, False)
    # a row of W loses half the smallest step of the 2^6 that the largest are brought to: 2^-31 of those
    dz, _, _ = rows.lmhead_grad(c.h, wide(c.w), c.lse.astype(np.float64), c.d_lse.astype(np.float64), c.d_zt.astype(np.float64), c.target, 1.0, 999)
    within(d_h, dh, bh + 2.0 ** -30 * np.abs(wide(c.w)).max() * np.abs(dz).sum(1, keepdims=True))


@pytest.mark.parametrize("M", [40, 300])
def test_a_row_that_is_not_finite_spoils_no_other_row(M):
    c = Case(M, 128, 400)
    c.d_lse[7], c.d_zt[9] = np.inf, np.nan
    c.target[9] = 3
    d_h = torch.zeros((M, 128), dtype=BF16, device=DEV)
    c.call(d_h, None)
    assert d_h[9].isnan().any() and not d_h[7].isfinite().all()
    good = np.delete(np.arange(M), [7, 9])
    for x in (c.d_lse, c.d_zt):
        x[[7, 9]] = 0.0
    dh, bh, _, _ = c.want(False, False)
    within(d_h[torch.from_numpy(good).to(DEV)], dh[good], bh[good])


@pytest.mark.parametrize("M,Dh,V", [(1, 64, 70), (67, 192, 300), (300, 320, 1000), (513, 64, 65)])
def test_target_logits_alone_are_exact(M, Dh, V):
    """Small whole numbers: every row of W and of hidden has to be there once, at its place."""
    rng = np.random.default_rng(M)
    h, w = rng.integers(-4, 5, (M, Dh)), rng.integers(-8, 9, (V, Dh))
    target, g = rng.integers(0, V, M), rng.integers(-3, 4, M)
    put = lambda x, t: torch.from_numpy(x.astype(np.float32)).to(t).to(DEV)
    d_h, d_w = torch.full((M, Dh), 7.0, dtype=F32, device=DEV), torch.full((V, Dh), 7.0, dtype=F32, device=DEV)
    lse = torch.full((M,), float("nan"), dtype=F32, device=DEV)
    how = dict(target=torch.from_numpy(target.astype(np.int32)).to(DEV), d_ztarget=put(g, F32), d_hidden=d_h, d_w=d_w)
    ws = torch.empty(dlm.lmhead_bwd_workspace_bytes(put(h, BF16), put(w, BF16), lse, **how), dtype=U8, device=DEV)
    dlm.lmhead_bwd(put(h, BF16), put(w, BF16), lse, workspace=ws, **how)
    want = np.zeros((V, Dh))
    np.add.at(want, target, g[:, None] * h)
    assert np.array_equal(wide(d_h), g[:, None] * w[target]) and np.array_equal(wide(d_w), want)


def test_probabilities_alone_are_exact():
    """W of zeros makes all probabilities exp(-lse); powers of two are exact in bf16, so d_w is a sum of whole numbers."""
    M, Dh, V = 130, 128, 333
    rng = np.random.default_rng(4)
    h, k, a = rng.integers(-3, 4, (M, Dh)), rng.integers(0, 5, M), 2.0 ** rng.integers(0, 3, M)
    put = lambda x, t: torch.from_numpy(x.astype(np.float32)).to(t).to(DEV)
    hidden, w, d_w = put(h, BF16), torch.zeros((V, Dh), dtype=BF16, device=DEV), torch.zeros((V, Dh), dtype=BF16, device=DEV)
    lse, d_lse = put(k * np.log(2.0), F32), put(a, F32)
    ws = torch.empty(dlm.lmhead_bwd_workspace_bytes(hidden, w, lse, d_lse=d_lse, d_w=d_w), dtype=U8, device=DEV)
    dlm.lmhead_bwd(hidden, w, lse, d_lse=d_lse, d_w=d_w, forbid_token=5, workspace=ws)
    want = ((a * 2.0 ** -k)[:, None] * h).sum(0)
    got = wide(d_w)
    assert (got[5] == 0).all() and (np.abs(np.delete(got, 5, 0) - want) <= H * np.abs(want)).all()


@pytest.mark.parametrize("columns", [256, 512, 1024])
def test_several_chunks_of_columns(columns):
    c = Case(200, 320, 1601, forbid=1600, gap=24)
    want = [torch.zeros((200, 320), dtype=F32, device=DEV), torch.zeros((1601, 320), dtype=BF16, device=DEV)]
    c.call(*want)
    dh, bh, dw, bw = c.want(True, False)
    dlm.set_option("lmhead_bwd_columns", columns)
    try:
        got = [torch.full_like(t, float("nan")) for t in want]
        c.call(*got)
    finally:
        dlm.set_option("lmhead_bwd_columns", 0)
    within(got[0], dh, bh)
    assert torch.equal(got[1], want[1])                 # each column is in one chunk


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,V", [(70, 333), (150, 333), (150, 1000), (300, 513)])
def test_whatever_the_workspace_held(M, V, dtype):
    c = Case(M, 128, V, forbid=2)
    lse, target, d_zt, d_lse = c.arrays()
    outs = []
    for fill in (0, 0x3f, 0x7f, 0x80, 0xff):             # as numbers small, some 2^30, and negative; as floating point 0.7, large and NaN
        d_h, d_w = (torch.full((n, 128), 7.0, dtype=dtype, device=DEV) for n in (M, V))
        how = dict(target=target, d_ztarget=d_zt, d_lse=d_lse, d_hidden=d_h, d_w=d_w, forbid_token=2)
        ws = torch.full((dlm.lmhead_bwd_workspace_bytes(c.hidden, c.w, lse, **how),), fill, dtype=U8, device=DEV)
        dlm.lmhead_bwd(c.hidden, c.w, lse, workspace=ws, **how)
        assert d_h.isfinite().all() and d_w.isfinite().all(), fill
        outs.append((d_h, d_w))
    assert all(torch.equal(a, b) for got in outs[1:] for a, b in zip(got, outs[0]))


def test_the_same_every_time_on_another_stream_and_from_a_graph():
    c = Case(140, 256, 900, rows_total=200, scatter=True, forbid=899)
    lse, target, d_zt, d_lse = c.arrays()
    idx, count = torch.from_numpy(c.idx).to(DEV), torch.tensor([140], dtype=I32, device=DEV)

    def call(d_h, d_w, ws, **kw):
        dlm.lmhead_bwd(c.hidden, c.w, lse, target=target, d_ztarget=d_zt, d_lse=d_lse, d_hidden=d_h, d_w=d_w, row_idx=idx, m_dev=count, forbid_token=899, out_scatter=True,
                       workspace=ws, **kw)

    outs = [(torch.zeros((200, 256), dtype=F32, device=DEV), torch.zeros((900, 256), dtype=BF16, device=DEV)) for _ in range(4)]
    size = dlm.lmhead_bwd_workspace_bytes(c.hidden, c.w, lse, target=target, d_ztarget=d_zt, d_lse=d_lse, d_hidden=outs[0][0], d_w=outs[0][1], row_idx=idx, m_dev=count,
                                          out_scatter=True)
    ws, ws2 = (torch.full((size,), 255, dtype=U8, device=DEV) for _ in range(2))
    call(*outs[0], ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call(*outs[1], ws2, stream=side)                     # beside the first
    side.synchronize()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs[0], outs[1]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(*outs[2], ws2)
    for live in (140, 64, 0, 1, 140):
        count.fill_(live)
        for k in (0, 2):
            outs[k][0].fill_(7.0)
            outs[k][1].fill_(7.0)
        ws2.fill_(255)
        graph.replay()
        call(*outs[0], ws)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs[0], outs[2])), live


def test_forward_and_backward_together():
    """lse and ztarget from lmhead_confidence, their gradient by this call, against differences of the 64-bit log-likelihood."""
    c = Case(48, 256, 1000, forbid=999)
    M = 48
    target = np.where((c.target >= 0) & (c.target < 999), c.target, 5).astype(np.int32)
    conf, lse, zt = (torch.zeros(M, dtype=F32, device=DEV) for _ in range(3))
    tok, tgt = torch.zeros(M, dtype=I32, device=DEV), torch.from_numpy(target).to(DEV)
    ws = torch.empty(dlm.lmhead_workspace_bytes(M, 1000), dtype=U8, device=DEV)
    dlm.lmhead_confidence(c.hidden, c.w, conf, tok, lse=lse, target=tgt, ztarget=zt, forbid_token=999, workspace=ws)
    d_h, d_w = torch.zeros((M, 256), dtype=F32, device=DEV), torch.zeros((1000, 256), dtype=F32, device=DEV)
    one = torch.ones(M, dtype=F32, device=DEV)
    how = dict(target=tgt, d_ztarget=one, d_lse=-one, d_hidden=d_h, d_w=d_w, forbid_token=999)
    big = torch.empty(dlm.lmhead_bwd_workspace_bytes(c.hidden, c.w, lse, **how), dtype=U8, device=DEV)
    dlm.lmhead_bwd(c.hidden, c.w, lse, workspace=big, **how)

    def value(h, w):
        z = h @ w.T
        z[:, 999] = -np.inf
        top = z.max(1)
        return (z[np.arange(M), target] - top - np.log(np.exp(z - top[:, None]).sum(1))).sum()

    h, w, r, step = c.h, wide(c.w), np.random.default_rng(0), 1e-5
    assert abs(float((zt - lse).double().sum()) - value(h, w)) < 1e-2
    for _ in range(4):
        u, v = r.standard_normal(h.shape), r.standard_normal(w.shape)
        dh, dw = (wide(d_h) * u).sum(), (wide(d_w) * v).sum()
        nh = (value(h + step * u, w) - value(h - step * u, w)) / (2 * step)
        nw = (value(h, w + step * v) - value(h, w - step * v)) / (2 * step)
        # 1e-4 of the gradient's norm is far above the errors of fp32 (see the bounds) and of the differences (1e-10 of the third derivative)
        assert abs(dh - nh) <= 1e-4 * np.linalg.norm(wide(d_h)) * np.linalg.norm(u) and abs(dw - nw) <= 1e-4 * np.linalg.norm(wide(d_w)) * np.linalg.norm(v)


def test_binding_checks():
    x, f, i = torch.zeros((4, 64), dtype=BF16, device=DEV), torch.zeros(4, dtype=F32, device=DEV), torch.zeros(4, dtype=I32, device=DEV)
    for kw, what in ((dict(d_lse=f[:3]), "entries"), (dict(d_lse=f, M=5), "more rows"), (dict(d_lse=f.double()), "dtype"), (dict(d_lse=f, d_hidden=x[:3]), "size"),
                     (dict(d_lse=f, row_idx=i.long()), "dtype"), (dict(d_lse=f, d_w=x[:, :32]), "size")):
        with pytest.raises(ValueError, match=what):
            dlm.lmhead_bwd(x, x, f, **dict(dict(d_w=x), **kw))
    with pytest.raises(ValueError, match="size"):
        dlm.lmhead_bwd(x, torch.zeros((4, 128), dtype=BF16, device=DEV), f, d_lse=f, d_hidden=x)
    with pytest.raises(dlm.DlmError) as e:
        dlm.lmhead_bwd(x, x, f, d_lse=f, d_hidden=x.clone())
    assert e.value.code == dlm.DLM_ERR_WORKSPACE
