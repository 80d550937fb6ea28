"""Attention over a paged cache, every shape of workgroup, alone and with shares, on inputs that separate right from nearly
right: probabilities whose roundings add up, huge scores (GPU)."""
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
@pytest.mark.parametrize("d", [64, 128])
def test_probabilities_keep_their_bits(form, d, e4m3):
    """Two kinds of keys whose values nearly cancel, so that what a probability loses is not averaged out: even ones with score 0 and value 1, odd ones with
    score -m / 8 in head m and value -x in column x.  Every score is exact, so a probability is within e = (4 m / 8 + 8) u of its own.  For the second product it is
    rounded, bf16: to 2^-15 of itself (two bf16 of it: half of its bits, and the nearest of what they leave, which is under 2^-7), with 128 rows a workgroup to 2^-8; 8-bit cache: to 2^-11
    or 2^-32 of the row's largest (fp16 of 128 times it or more)."""
    lens = [40] if form[0] in (1, 4) else [900, 64]
    c = Case(lens, 3, 16, 2, d, 16, e4m3)
    m = torch.arange(16, device=DEV) % 8 + 1.0 + torch.arange(16, device=DEV) // 8 * 8
    c.q.zero_()
    c.q[..., 0] = m
    x = torch.tensor([(1 + i / 8) * 2 ** k for k in range(3) for i in range(8)])
    values = -x[torch.arange(d) % len(x)]
    for b, n in enumerate(lens):
        odd = (torch.arange(n) % 2)[:, None]
        fill(c, 0, b, np.arange(n), -odd.expand(n, d).float())
        fill(c, 1, b, np.arange(n), torch.where(odd == 1, values, torch.ones(d)))
    if e4m3:
        c.scales[0].fill_(1.0), c.scales[1].fill_(1.0)
    run(form, c, scale=0.125)
    out, lse, mag, _ = heads.paged_attention(wide(c.q), *c.values(), c.table.cpu().numpy(), lens, scale=0.125)
    e = (4 * m.cpu().numpy() / 8 + 8) * U
    p = 2.0 ** -11 + max(lens) * 2.0 ** -32 * 7.5 if e4m3 else H if form[0] == 3 else 2.0 ** -15 + 2.0 ** -23
    bound = (p + 2 * e[None, None, :, None] + 2 * max(lens) * U) * mag * (1 + H) + H * np.abs(out) * (1 + H)
    err = np.abs(wide(c.out) - out)
    assert (err <= bound).all(), (err / bound).max()
    assert (np.abs(wide(c.lse) - lse) <= e[None, :, None] + 2 * max(lens) * U + 4 * U * np.abs(lse)).all()


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
