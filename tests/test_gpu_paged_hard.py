"""Attention over a paged cache, every shape of workgroup, alone and with shares, on inputs that separate right from nearly right: probabilities whose
roundings add up, scores that rise from tile to tile or are huge, absent pages, what is not finite (GPU)."""
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
CAUSAL = dict(mask_mode=dlm.MASK_BLOCK_CAUSAL, block_size=1)


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
def test_many_small_probabilities(form, e4m3):
    """One key of score 0 and value 0 and 20000 of score -18 and value 1: each has 2^-26 of the largest probability, in fp16 a number without its full 11 bits, and their
    sum decides.  Bound as above: 2^-32 of the largest for each of them, 2 e + 2 n u and the output's rounding of the sum."""
    n = 20001
    c = Case([n], 3, 8, 2, 64, 64, e4m3)
    if e4m3:
        c.scales[0].fill_(1.0), c.scales[1].fill_(1.0)
    first, value = torch.full((n, 1), -18.0), torch.ones(n, 64)
    first[11111], value[11111] = 0, 0
    fill(c, 0, 0, np.arange(n), first)
    fill(c, 1, 0, np.arange(n), value)
    c.q.zero_()
    c.q[..., 0] = 1
    run(form, c, scale=1.0)
    small = 20000 * np.exp(-18.0)
    want, e = small / (1 + small), (4 * 18 + 8) * U
    p = n * 2.0 ** -32 if e4m3 else H * want if form[0] == 3 else 2.0 ** -14 * want
    assert (np.abs(wide(c.out) - want) <= p + (2 * e + 2 * n * U) * want + H * want * (1 + H)).all()
    assert (np.abs(wide(c.lse) - np.log1p(small)) <= e + 2 * n * U).all()


# whole numbers that both types of cache hold
LEVELS = list(range(-16, 17)) + list(range(18, 33, 2)) + list(range(36, 65, 4))


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("Lq", [2, 9])
def test_scores_that_rise_from_tile_to_tile(form, Lq, e4m3):
    """Every tile's scores lie 12 above those of the tile before for some rows, below for others, in a random order for a second sequence: what has been summed up is scaled down again and again."""
    n = 32 * len(LEVELS) - 7
    c = Case([n, n], Lq, 8, 2, 64, 16, e4m3)
    if e4m3:
        c.scales[0].fill_(1.0), c.scales[1].fill_(1.0)
    for b in range(2):
        level = torch.tensor(LEVELS, dtype=torch.float32)
        if b:
            level = level[torch.from_numpy(c.rng.permutation(len(LEVELS)))]
        fill(c, 0, b, np.arange(n), torch.stack([level[torch.arange(n) // 32], torch.from_numpy(c.rng.standard_normal(n)).float()], 1))
    c.q[..., 2:] = 0
    c.q[..., 1] = 1
    c.q[..., 0] = torch.tensor([12.0, -12.0, 0.0, 6.0, 12.0, 0.5, -12.0, 12.0], device=DEV)
    for mask in ({}, CAUSAL):
        run(form, c, scale=1.0, **mask)
        c.check(**mask, scale=1.0)


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


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("page", [16, 64])
def test_absent_pages_all_over(form, page, e4m3):
    """A quarter of the pages of long sequences is not there: every parity of tile, either half of one, first and last ones, a sequence without any."""
    c = Case([1500, 1490, 700, 300], 9, 8, 2, 128, page, e4m3)
    gone = c.rng.random(c.table.shape) < 0.25
    gone[0, 0] = gone[0, 1500 // page] = gone[1, 1] = True
    gone[3] = True
    lost = torch.from_numpy(np.where(c.rng.random(gone.shape) < 0.5, -1, 1 << 30).astype(np.int32)).to(DEV)
    c.table.copy_(torch.where(torch.from_numpy(gone).to(DEV), lost, c.table))
    for mask in ({}, dict(mask_mode=dlm.MASK_BLOCK_CAUSAL, block_size=4)):
        run(form, c, **mask)
        c.check(**mask)


@pytest.mark.parametrize("e4m3", [False, True])
def test_nan_where_nobody_looks(form, e4m3):
    """NaN in rows behind the end of a sequence, in pages that nobody owns, and in keys that a causal mask hides."""
    c = Case([1301, 21, 64, 700, 0], 9, 8, 2, 64, 32, e4m3)
    owned = torch.zeros(c.pages[0].shape[0], 32, dtype=torch.bool, device=DEV)
    for b, n in enumerate(c.lengths):
        for t in range(n):
            owned[where(c, b, t)] = True
    for x in c.pages:
        x.view(torch.uint8 if e4m3 else torch.int16).transpose(1, 2)[~owned] = 0x7f if e4m3 else 0x7fc0
    for mask in ({}, CAUSAL):
        run(form, c, **mask)
        c.check(**mask)
    run(form, c, **CAUSAL)
    before = c.out.clone(), c.lse.clone()
    page, row = where(c, 0, 1296)                   # the key of query row 4
    raw = c.pages[0].view(torch.uint8 if e4m3 else torch.int16)
    raw[page, 1, row, 7] = 0x7f if e4m3 else 0x7fc0
    run(form, c, **CAUSAL)
    assert c.out[0, 4:, 4:].isnan().all() and c.lse[0, 4:, 4:].isnan().all()
    c.out[0, 4:, 4:], c.lse[0, 4:, 4:] = before[0][0, 4:, 4:], before[1][0, 4:, 4:]
    assert torch.equal(c.out, before[0]) and torch.equal(c.lse, before[1])


def test_what_is_not_finite_stays_where_it_is(form):
    """NaN in a key reaches every row of its KV head, NaN or an infinity in a value its column only, NaN in a query its row; scores of -inf count as not seen, all of a
    row's or those of some tiles."""
    c = Case([1000, 1000, 1000, 1000, 1000], 9, 8, 2, 64, 16)
    page, row = where(c, 0, 707)
    c.pages[0][page, 0, row, 3] = float("nan")
    page, row = where(c, 1, 209)
    c.pages[1][page, 0, row, 5], c.pages[1][page, 1, row, 6] = float("nan"), float("inf")
    c.q[2:4, ..., 0] = 1.0
    for b, hidden in ((2, range(1000)), (3, [*range(0, 40), *range(100, 612), 999])):
        for t in hidden:
            page, row = where(c, b, t)
            c.pages[0][page, :, row, 0] = float("-inf")
    c.q[4, 3, 2, 9] = float("nan")
    run(form, c)
    out, lse = c.out, c.lse
    assert out[0, :, :4].isnan().all() and lse[0, :4].isnan().all()
    assert out[1, :, :4, 5].isnan().all() and (out[1, :, 4:, 6] == float("inf")).all()
    assert (out[2] == 0).all() and (lse[2] == -float("inf")).all()
    assert out[4, 3, 2].isnan().all() and lse[4, 2, 3].isnan()
    # the rest as without them
    clean = Case([1000, 1000, 1000, 1000, 1000], 9, 8, 2, 64, 16)
    clean.q[2:4, ..., 0] = 1.0
    clean.q[4, 3, 2, 9] = 0
    want, want_lse, mag, top = heads.paged_attention(wide(clean.q), *clean.values(), clean.table.cpu().numpy(), clean.lengths)
    k, v = clean.values()
    seen = [t for t in range(1000) if not (t < 40 or 100 <= t < 612 or t == 999)]
    at = [where(c, 3, t) for t in seen]
    for i in range(9):
        for h in range(8):
            s = np.array([k[p, h // 4, r] for p, r in at]) @ wide(clean.q)[3, i, h] / 8
            p = np.exp(s - s.max())
            vv = np.array([v[pg, h // 4, r] for pg, r in at])
            want_lse[3, h, i] = s.max() + np.log(p.sum())
            want[3, i, h], mag[3, i, h] = p @ vv / p.sum(), p @ np.abs(vv) / p.sum()
    e = 2 * (64 + 16) * U * top + 8 * U
    bound = (H + 2 * np.moveaxis(e, 1, 2)[..., None] + 2000 * U) * mag + H * np.abs(want) * (1 + H)
    fine = np.ones(want.shape, dtype=bool)
    fine[0, :, :4] = fine[1, :, :4, 5] = fine[1, :, 4:, 6] = fine[2] = fine[4, 3, 2] = False
    assert (np.abs(wide(out) - want)[fine] <= bound[fine]).all()
    assert (np.abs(wide(lse) - want_lse)[3] <= e[3] + 2000 * U + 4 * U * np.abs(want_lse[3])).all()


def test_shares_are_taken_where_they_are_asked_for():
    """n workgroups share keys with 32 and 128 rows a workgroup (at least 8 tiles each), never with 16 rows."""
    c = Case([4000, 3000], 2, 8, 2, 64, 16)
    given = (c.q, c.out, *c.pages, c.table, c.lens)
    try:
        for shape, some in ((1, False), (2, True), (3, True), (4, False)):
            dlm.set_option("paged_shape", shape)
            sizes = []
            for n in (1, 7, 10 ** 4):
                dlm.set_option("paged_shares", n)
                sizes.append(dlm.paged_attn_workspace_bytes(*given))
                c.run()
                c.check()
            assert all((s > 0) == some for s in sizes)
            if some:                                # 125 tiles of 4 row groups: 62 shares at most
                rows = 32 if shape == 2 else 128
                assert sizes == [2 * s * rows * 66 * 4 + 2 * 4 * 4 for s in (1, 7, 62)]
    finally:
        dlm.set_option("paged_shape", 0)
        dlm.set_option("paged_shares", 0)
