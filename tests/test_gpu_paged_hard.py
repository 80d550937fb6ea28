"""Attention over a paged cache, every shape of workgroup, alone and with shares, on inputs that separate right from nearly
right: huge scores (GPU)."""
import numpy as np
import pytest
import torch

from oracle import heads
from paper_2604_04215_amd import binding as dlm
from gpu_util import DEV
from test_gpu_paged_attn import H, U, Case, wide

pytestmark = pytest.mark.gpu

# (paged_shape, paged_shares): 16, 32, 128, 16 rows; 16 rows are never shared out
FORMS = [(0, 0), (1, 0), (4, 0), (2, -1), (2, 5), (2, 40), (3, -1), (3, 5), (3, 40)]


@pytest.fixture(params=FORMS, ids=lambda f: "shape%d-shares%d" % f)
def form(request):
    dlm.set_option("paged_shape", request.param[0])
    dlm.set_option("paged_shares", request.param[1])
    yield request.param
    dlm.set_option("paged_shape", 0)
    dlm.set_option("paged_shares", 0)


def run(form, c, **kw):
    """One call, which shares its keys where that is what the form says."""
    n = c.run(**kw)
    assert (n > 0) == (form[1] > 0) or form == (0, 0)


def where(c, b, t):
    """Page and row of token t."""
    page = c.pages[0].shape[2]
    return int(c.table[b, t // page]), t % page


def fill(c, which, b, rows, values):
    """Rows of sequence b for all its KV heads: values [len(rows), ...] of entries `values.shape[-1]` from the first on."""
    page = c.pages[0].shape[2]
    rows = torch.as_tensor(np.asarray(rows), device=DEV)
    at = c.table[b].long()[rows // page], rows % page
    x = c.pages[which].float()
    x.transpose(1, 2)[at[0], at[1], :, :values.shape[-1]] = values.to(DEV).float()[:, None]
    c.pages[which].copy_(x.to(c.pages[which].dtype))


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("power", [21, 25, 31, 40, 60])
def test_huge_scores(form, power, e4m3):
    """Scores of 1.57 2^21 to 1.57 2^60, all finite: the largest decides (two alike: their mean), and rows beside it whose scores are zero have the mean of all."""
    n = 700
    c = Case([n], 5, 8, 2, 64, 16, e4m3)
    if e4m3:
        c.scales[0].fill_(1.0), c.scales[1].fill_(1.0)
    first = torch.zeros(n, 1)
    first[[45, 601]] = 1.0
    first[[333, 699]] = -1.0
    fill(c, 0, 0, np.arange(n), first)
    c.q.zero_()
    q0 = torch.tensor([1.0, 0.0, -1.0, 0.0, 1.0, -1.0, 1.0, 0.0], device=DEV) * 201 * 2.0 ** (power - 7)
    c.q[..., 0] = q0
    run(form, c, scale=1.0)
    _, v = c.values()
    rows = np.stack([v[where(c, 0, t)[0], :, where(c, 0, t)[1]] for t in range(n)])                 # [n, Hkv, d]
    for h in range(8):
        picked = rows[[45, 601] if q0[h] > 0 else [333, 699] if q0[h] < 0 else list(range(n)), h // 4]
        want, mag = picked.mean(0), np.abs(picked).mean(0)
        got = wide(c.out)[0, :, h]
        assert (np.abs(got - want) <= (2.0 ** -11 + 2 * n * U + 32 * U) * mag + H * np.abs(want) * (1 + H)).all()
        lse = np.log(len(picked)) + abs(float(q0[h]))
        assert (np.abs(wide(c.lse)[0, h] - lse) <= 8 * U * lse + 2 * n * U).all()
