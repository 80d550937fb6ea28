"""The LM head's gradient row by row: every row of d_w and of d_hidden by its own size, however small beside the others (GPU).

Bounds, u = 2^-24, h = 2^-8 (half steps of fp32 and bf16), t = 2^-11 (of fp16).  Logits, probabilities and sums as in test_gpu_lmhead_bwd.py.  What is stored of dz is
t |dz| off, or, of numbers far below the largest of their kind:
  for d_hidden  2^-39 of the row's |d_lse| + |d_ztarget| (inv_t included) times the spread of W's rows, which is below 2^10 here: 2^-28;
  for d_w       2^-22 of the largest |dz| 2^e of the column, e the exponent of the largest entry of its hidden row; of which, with |h| < 2^(e + 1), the M rows
                together make at most 2 M 2^-22 of that largest.  It is t of it, for which its own row already stands, up to M = 2^10.
(Up to 128 rows two bf16 terms: h^2 |dz| and nothing beside it.  The library by itself takes them for sizes like these up to 1024 rows; here it is told not to.)"""
import numpy as np
import pytest
import torch

from oracle import rows
from paper_2604_04215_amd import binding as dlm
from gpu_util import DEV, GuardedWorkspace

pytestmark = pytest.mark.gpu
U, H, T = 2.0 ** -24, 2.0 ** -8, 2.0 ** -11
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


@pytest.fixture(autouse=True)
def few():
    dlm.set_option("lmhead_bwd_few", 128)
    yield
    dlm.set_option("lmhead_bwd_few", 0)


def wide(t):
    return t.detach().double().cpu().numpy()


def put(x, t=BF16):
    return torch.from_numpy(np.ascontiguousarray(x).astype(np.int32 if t == I32 else np.float32)).to(t).to(DEV)


def s(K):
    return 2 * U * (16 + K / 16)


class Rows:
    def __init__(self, hidden, w, target, d_zt, d_lse, lse_up=0.0, forbid=-1):
        self.hidden, self.w, self.target, self.forbid = put(hidden), put(w), target.astype(np.int32), forbid
        self.h, self.w64 = wide(self.hidden), wide(self.w)
        self.M, self.Dh, self.V = *self.h.shape, len(self.w64)
        z = self.z = self.h @ self.w64.T
        if forbid >= 0:
            z[:, forbid] = -np.inf
        top = z.max(1, keepdims=True)
        self.lse = ((top + np.log(np.exp(z - top).sum(1, keepdims=True)))[:, 0] + lse_up).astype(np.float32)
        self.d_zt, self.d_lse = (np.asarray(x, np.float32) for x in (d_zt, d_lse))

    def call(self, d_hidden=True, d_w=True):
        got = [torch.full((n, self.Dh), float("nan"), dtype=BF16, device=DEV) if on else None for n, on in ((self.M, d_hidden), (self.V, d_w))]
        lse = put(self.lse, F32)
        how = dict(target=put(self.target, I32), d_ztarget=put(self.d_zt, F32), d_lse=put(self.d_lse, F32), d_hidden=got[0], d_w=got[1], forbid_token=self.forbid)
        ws = GuardedWorkspace(dlm.lmhead_bwd_workspace_bytes(self.hidden, self.w, lse, **how))
        ws.ws.fill_(255)
        dlm.lmhead_bwd(self.hidden, self.w, lse, workspace=ws.ws, **how)
        ws.check()
        return got

    def check(self, d_hidden, d_w):
        lse, a, c = (x.astype(np.float64) for x in (self.lse, self.d_lse, self.d_zt))
        dz, dh, dw = rows.lmhead_grad(self.h, self.w64, lse, a, c, self.target, 1.0, self.forbid)
        finite = np.where(np.isinf(self.z), 0.0, self.z)
        e = s(self.Dh) * (np.abs(self.h) @ np.abs(self.w64).T) + 4 * U * (np.abs(finite) + np.abs(lse)[:, None])
        off = np.abs(a)[:, None] * np.exp(self.z - lse[:, None]) * (np.expm1(e) + 8 * U) + 4 * U * np.abs(dz) + 2.0 ** -126
        # what a target's sum of two terms loses is of the terms, not of the sum
        live = (self.target >= 0) & (self.target < self.V) & (self.target != self.forbid)
        at = np.flatnonzero(live), self.target[live]
        off[at] += 2 * U * np.abs(c[live])
        few, size, ah, aw = self.M <= 128, np.abs(dz), np.abs(self.h), np.abs(self.w64)
        if d_hidden is not None:
            floor = 0.0 if few else 2.0 ** -28 * (np.abs(a) + np.abs(c))[:, None]
            bound = (off * 1.01 + (H * H if few else T) * size + floor) @ aw + (s(2 * self.V) + 128 * U) * ((size + off) @ aw)
            err = np.abs(wide(d_hidden) - dh)
            assert (err <= H * np.abs(dh) + bound * 1.01).all(), (err / (H * np.abs(dh) + bound)).max()
        if d_w is None:
            return
        top = np.abs(self.h).max(1)
        e2 = np.where(top > 0, 2.0 ** np.floor(np.log2(np.where(top > 0, top, 1))), 0.0)
        largest = ((size + off) * e2[:, None]).max(0)
        floor = 0.0 if few else 2 * self.M * 2.0 ** -22 * largest[:, None]
        bound = (off * 1.01 + (H * H if few else T) * size).T @ ah + s(2 * self.M) * ((size + off).T @ ah) + floor
        err = np.abs(wide(d_w) - dw)
        assert (err <= H * np.abs(dw) + bound * 1.01 + 2.0 ** -126).all(), (err / (H * np.abs(dw) + bound + 1e-300)).max()
        # in the norm of each row: the rounding of bf16, at most h, and what off allows
        norm = lambda x: np.sqrt((x * x).sum(1))
        rel, want = norm(wide(d_w) - dw), norm(dw)
        assert (rel <= H * want + norm((off * 1.01).T @ ah)).all(), ((rel / (want + 1e-300)).max(), (rel > H * want).sum())


MS = [100, 129, 300, 700]


def draws(M, Dh, V, seed):
    rng = np.random.default_rng(seed)
    return rng, rng.standard_normal((M, Dh)), rng.standard_normal((V, Dh))


@pytest.mark.parametrize("only", [None, "d_hidden", "d_w"])
@pytest.mark.parametrize("M", MS)
def test_wide_logits(M, only):
    """Logits of size 12: most tokens are unlikely in every row."""
    rng, h, w = draws(M, 256, 3000, M)
    g = rng.uniform(0.1, 1, M)
    c = Rows(h, w * 0.75, rng.integers(0, 2999, M), g, -g, forbid=2999)
    c.check(*c.call(d_hidden=only != "d_w", d_w=only != "d_hidden"))


@pytest.mark.parametrize("gap", [20, 40, 70])
@pytest.mark.parametrize("M", MS)
def test_confident_rows(M, gap):
    """The target's logit that far above the others in every row."""
    rng, h, w = draws(M, 256, 1003, M + gap)
    w *= 3.0 / 16
    target, g = rng.integers(0, 1002, M), rng.uniform(0.5, 2, M)
    pull = w[target]
    h += pull / (pull * pull).sum(1, keepdims=True) * (gap - (h * pull).sum(1, keepdims=True))
    c = Rows(h, w, target, -g, g, forbid=1002)
    c.check(*c.call())


@pytest.mark.parametrize("M", [300, 700, 1000])
def test_columns_that_some_rows_alone_make_large(M):
    """Probabilities of one stretch of the rows 2^-20 to 2^-90 of those of another, and gradients of very different size in between."""
    rng, h, w = draws(M, 128, 700, M)
    up = np.repeat(rng.permutation(np.arange(-(-M // 30)) % 4 * 14.0 + 0.1), 30)[:M]
    g = rng.uniform(0.5, 2, M) * 2.0 ** -rng.integers(0, 12, M)
    c = Rows(h, w * 0.2, rng.integers(-1, 40, M), g, -g, lse_up=up)
    c.check(*c.call())


@pytest.mark.parametrize("M", MS)
def test_gradients_of_targets_alone_keep_every_size(M):
    """Without probabilities a row of d_w is one gradient times one hidden row, of which every entry has its own bits, whatever its size."""
    rng, h, w = draws(M, 128, 1000, 7 * M)
    h *= 2.0 ** rng.integers(-14, 1, (M, 128)) * 2.0 ** rng.integers(-40, 40, (M, 1))
    g = rng.standard_normal(M) * 2.0 ** rng.integers(-40, 1, M)
    c = Rows(h, np.zeros((1000, 128)), rng.permutation(1000)[:M], g, np.zeros(M))
    got = wide(c.call(d_hidden=False)[1])
    want = np.zeros((1000, 128))
    want[c.target] = c.d_zt.astype(np.float64)[:, None] * c.h
    # the gradient is rounded to 11 bits (t), the result to 8 (h)
    assert (np.abs(got - want) <= (H + T) * 1.01 * np.abs(want)).all()


@pytest.mark.parametrize("M", MS)
@pytest.mark.parametrize("power", [-40, -90])
def test_gradients_of_small_hidden_rows(M, power):
    """Every other hidden row nearly zero: its gradient is not."""
    rng, h, w = draws(M, 128, 500, 3 * M)
    h[::2] *= 2.0 ** power
    g = rng.uniform(0.5, 2, M)
    c = Rows(h, w * 0.3, rng.integers(0, 500, M), g, -g)
    c.check(*c.call())
