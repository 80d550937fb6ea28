"""Attention over a paged cache against the 64-bit definition (GPU).

Bound of an output entry, u = 2^-24, h = 2^-8: a score is a sum of d products (error under (d + 8) u times sum |q||k| scale = S), so a
probability's relative error is under e = 2 (d + 16) u S + 8 u; it is rounded to bf16 (h); the sums over the keys add n u; the output is rounded
to bf16: (h + 2 e + 2 n u) sum_j p_j |v_j| + h |o|.  The log-sum-exp's: e + 2 n u + 4 u |lse|."""
import numpy as np
import pytest
import torch

from oracle import heads
from paper_2604_04215_amd import binding as dlm
from gpu_util import DEV, GuardedWorkspace

pytestmark = pytest.mark.gpu
U, H = 2.0 ** -24, 2.0 ** -8
BF16, F32, I32, E4M3 = torch.bfloat16, torch.float32, torch.int32, torch.float8_e4m3fn


def wide(t):
    return t.detach().double().cpu().numpy()


class Case:
    def __init__(self, lens, Lq, Hq, Hkv, d, page, e4m3=False, q_len=None, spare=3, seed=0, token_major=False):
        rng = self.rng = np.random.default_rng(seed + 31 * sum(lens) + Lq + d + page)
        B = len(lens)
        counts = [-(-n // page) for n in lens]
        n_pages = sum(counts) + spare
        order, at = rng.permutation(n_pages), 0
        table = np.full((B, max(counts + [1])), -7, dtype=np.int32)          # entries behind a sequence's end: never looked at
        for b, m in enumerate(counts):
            table[b, :m] = order[at:at + m]
            at += m
        shape = (n_pages, page, Hkv, d) if token_major else (n_pages, Hkv, page, d)
        std = 60.0 if e4m3 else 1.0
        self.pages = [torch.from_numpy(rng.standard_normal(shape).astype(np.float32) * std).to(E4M3 if e4m3 else BF16).to(DEV) for _ in range(2)]
        if token_major:
            self.pages = [x.transpose(1, 2) for x in self.pages]
        self.scales = [torch.from_numpy((0.012 + 0.01 * rng.random(Hkv)).astype(np.float32)).to(DEV) if e4m3 else None for _ in range(2)]
        self.q = torch.from_numpy(rng.standard_normal((B, Lq, Hq, d)).astype(np.float32)).to(BF16).to(DEV)
        self.table, self.lens = torch.from_numpy(table).to(DEV), torch.tensor(lens, dtype=I32, device=DEV)
        self.q_len = None if q_len is None else torch.tensor(q_len, dtype=I32, device=DEV)
        self.out, self.lse = torch.full_like(self.q, 7.0), torch.full((B, Hq, Lq), 7.0, device=DEV)
        self.lengths = lens

    def run(self, split=True, **kw):
        how = dict(q_len=self.q_len, lse=self.lse, k_scale=self.scales[0], v_scale=self.scales[1], **kw)
        given = (self.q, self.out, *self.pages, self.table, self.lens)
        n = dlm.paged_attn_workspace_bytes(*given, **how) if split else 0
        ws = GuardedWorkspace(n) if n else None
        dlm.paged_attn(*given, workspace=None if ws is None else ws.ws, **how)
        torch.cuda.synchronize()
        if ws is not None:
            ws.check()
        return n

    def values(self):
        k, v = (wide(x) for x in self.pages)
        if self.scales[0] is not None:
            k, v = (x * wide(s)[None, :, None, None] for x, s in zip((k, v), self.scales))
        return k, v

    def check(self, mask_mode=0, block_size=0, scale=None):
        q_len = None if self.q_len is None else self.q_len.cpu().numpy()
        out, lse, mag, top = heads.paged_attention(wide(self.q), *self.values(), self.table.cpu().numpy(), np.maximum(self.lengths, 0), q_len,
                                                   block_size if mask_mode else 0, scale)
        compare(self, out, lse, mag, top)


def compare(c, out, lse, mag, top):
    n, d = max(max(c.lengths), 1), c.q.shape[-1]
    got, got_lse, left = wide(c.out), wide(c.lse), np.isnan(out)
    assert (got[left] == 7.0).all() and (got_lse[np.isnan(lse)] == 7.0).all()                # rows behind the last one
    e = 2 * (d + 16) * U * top + 8 * U
    bound = (H + 2 * np.moveaxis(e, 1, 2)[..., None] + 2 * n * U) * mag + H * np.abs(out) * (1 + H) + 2.0 ** -133
    assert (np.abs(got - out)[~left] <= bound[~left]).all(), (np.abs(got - out)[~left] / (bound[~left] + 1e-300)).max()
    live = np.isfinite(lse)
    assert np.array_equal(got_lse[lse == -np.inf], lse[lse == -np.inf])
    assert (np.abs(got_lse[live] - lse[live]) <= (e + 2 * n * U)[live] + 4 * U * np.abs(lse[live])).all()


SHAPES = [([1], 1, 1, 1, 64, 16), ([1, 31, 32, 33], 1, 14, 2, 64, 16), ([400, 17, 3], 1, 32, 8, 128, 64), ([0, 5, 64, 65], 1, 4, 4, 128, 16),
          ([130, 700], 4, 32, 8, 128, 32), ([97, 256, 255], 32, 4, 4, 64, 256), ([300, 40], 32, 28, 4, 128, 128), ([2500], 1, 4, 2, 128, 16), ([1900, 33], 7, 6, 2, 64, 64),
          ([3, 40], 8, 4, 2, 64, 16)]


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("lens,Lq,Hq,Hkv,d,page", SHAPES)
def test_full_mask(lens, Lq, Hq, Hkv, d, page, e4m3):
    c = Case(lens, Lq, Hq, Hkv, d, page, e4m3)
    for split in (True, False):
        c.run(split)
        c.check()


@pytest.mark.parametrize("bs", [1, 4, 32])
@pytest.mark.parametrize("lens,Lq,Hq,Hkv,d,page", SHAPES)
def test_block_causal(lens, Lq, Hq, Hkv, d, page, bs):
    """(sequences shorter than Lq have rows in front of position 0, which see nothing)"""
    c = Case(lens, Lq, Hq, Hkv, d, page, e4m3=bs == 4)
    c.run(mask_mode=dlm.MASK_BLOCK_CAUSAL, block_size=bs)
    c.check(dlm.MASK_BLOCK_CAUSAL, bs)


@pytest.mark.parametrize("mask", [{}, dict(mask_mode=dlm.MASK_BLOCK_CAUSAL, block_size=4)])
def test_fewer_rows_than_the_batch_has(mask):
    c = Case([50, 1200, 9, 300], 9, 8, 2, 128, 32, q_len=[9, 0, 3, 8], token_major=True)
    c.run(**mask)
    c.check(**mask)
    c = Case([50, 1200], 2, 4, 4, 64, 16, q_len=[-3, 99])            # taken as 0 and Lq
    c.run(**mask)
    c.q_len = c.q_len.clamp(0, 2)
    c.check(**mask)


@pytest.fixture
def options():
    yield dlm.set_option
    dlm.set_option("paged_shape", 0)
    dlm.set_option("paged_shares", 0)


@pytest.mark.parametrize("shares", [0, -1, 1, 2, 7, 64, 1000])
@pytest.mark.parametrize("shape", [1, 2, 3, 4])
@pytest.mark.parametrize("d", [64, 128])
def test_every_shape_of_workgroup(options, shape, shares, d):
    """16, 32 and 128 rows a workgroup, keys dealt out to few workgroups and to more than there are, for few rows and many, every mask and type."""
    options("paged_shape", shape)
    options("paged_shares", shares)
    for i, (lens, Lq, Hq, Hkv, page) in enumerate([([1, 40, 333], 1, 4, 2, 16), ([700, 95], 5, 14, 2, 64), ([200, 513], 33, 8, 2, 32), ([1500], 3, 5, 1, 128)]):
        for e4m3 in (False, True):
            for mask in ({}, dict(mask_mode=dlm.MASK_BLOCK_CAUSAL, block_size=(1, 4, 32, 7)[i])):
                c = Case(lens, Lq, Hq, Hkv, d, page, e4m3, q_len=[max(Lq - 2 * k, 0) for k in range(len(lens))] if i % 2 else None, seed=i)
                c.run(**mask)
                c.check(**mask)


@pytest.mark.parametrize("shape", [1, 2, 3, 4])
def test_more_than_32_tiles_a_wavefront(options, shape):
    """The look-ups of pages go on past the first 32 tiles."""
    options("paged_shape", shape)
    options("paged_shares", -1)
    c = Case([9001, 4097, 31], 1, 2, 1, 64, 16)
    assert c.run() == 0
    c.check()


@pytest.mark.parametrize("B", [1, 255, 300, 700])
def test_many_sequences_share_the_workgroups(options, B):
    """Lengths from nothing to long, sequences without rows among them, more sequences than a workgroup has threads."""
    options("paged_shape", 2)
    options("paged_shares", 64)
    rng = np.random.default_rng(B)
    lens = [int(x) for x in rng.integers(0, 60, B)]
    lens[-1], lens[B // 2] = 0, 700
    q_len = [int(x) for x in rng.integers(0, 3, B)]
    for mask in ({}, dict(mask_mode=dlm.MASK_BLOCK_CAUSAL, block_size=1)):
        c = Case(lens, 2, 2, 1, 64, 16, q_len=q_len)
        assert c.run(**mask) > 0
        c.check(**mask)
    c.q_len.zero_()                                   # nobody asks
    c.out.fill_(7.0), c.lse.fill_(7.0)
    c.run()
    assert (c.out == 7).all() and (c.lse == 7).all()


def test_long_sequence_split_and_not():
    """Enough keys for many stretches; both sides of a stretch's border; lengths outside [0, max_kv_len] are clamped."""
    for lens in ([9000], [8191, 12, 0, 6000], [70000]):
        c = Case(lens, 1, 8, 2, 64, 64)
        assert c.run() > 0
        c.check()
    c = Case([3000, 100], 1, 4, 4, 64, 16)
    c.lens[0], c.lens[1] = 1 << 30, -5
    c.run(max_kv_len=2900)
    c.lengths = [2900, 0]
    c.check()


def test_no_keys_at_all():
    """Tables without entries, caches without pages, sequences without tokens: zeros, and a log-sum-exp of -inf."""
    c = Case([0, 0], 2, 4, 2, 64, 16)
    for table, pages in ((c.table[:, :0], c.pages), (c.table, [x[:0] for x in c.pages]), (c.table, c.pages)):
        c.out.fill_(7.0), c.lse.fill_(7.0)
        c.lens.fill_(5 if table.shape[1] else 0)
        if pages is c.pages:
            c.lens.zero_()
        dlm.paged_attn(c.q, c.out, *pages, table, c.lens, lse=c.lse)
        assert (c.out == 0).all() and (c.lse == -float("inf")).all()
    dlm.paged_attn(c.q[:0], c.out[:0], *c.pages, c.table[:0], c.lens[:0])
    dlm.paged_attn(c.q[:, :0], c.out[:, :0], *c.pages, c.table, c.lens)


def test_absent_pages():
    """Pages outside [0, n_pages): their keys are not there, wherever they lie."""
    c = Case([200, 64, 40], 2, 4, 2, 128, 16)
    c.table[0, 0], c.table[0, 3], c.table[0, 12], c.table[1] = -1, 1 << 30, c.pages[0].shape[0], -1
    c.run()
    c.check()


@pytest.mark.parametrize("split", [True, False])
def test_garbage_behind_the_end_and_in_nobodys_pages(split):
    for e4m3 in (False, True):
        c = Case([1300, 21, 64], 3, 4, 2, 64, 32, e4m3)
        owned = torch.zeros(c.pages[0].shape[0], 32, dtype=torch.bool, device=DEV)
        for b, n in enumerate(c.lengths):
            for t in range(n):
                owned[c.table[b, t // 32], t % 32] = True
        for x in c.pages:
            raw = x.view(torch.uint8 if e4m3 else torch.int16)
            raw.transpose(1, 2)[~owned] = 0x7f if e4m3 else 0x7fc0              # NaN
        c.run(split)
        c.check()


def test_what_is_not_finite():
    """NaN in a key or value reaches the rows that see it; scores of -inf count as not seen."""
    c = Case([40, 40, 40, 40], 1, 2, 1, 64, 16)
    at = lambda b, t: (int(c.table[b, t // 16]), 0, t % 16)
    c.pages[0][at(0, 7)][3] = float("nan")
    c.pages[1][at(1, 9)][5] = float("nan")
    c.q[2] = 1.0
    for t in range(40):
        c.pages[0][at(2, t)][0] = float("-inf")
    c.run()
    assert c.out[0].isnan().all() and c.lse[0].isnan().all()
    assert c.out[1, ..., 5].isnan().all() and c.out[1, ..., 6:].isfinite().all()
    assert (c.out[2] == 0).all() and (c.lse[2] == -float("inf")).all()
    assert c.out[3].isfinite().all()


@pytest.mark.parametrize("shape", [1, 2, 3, 4])
def test_every_8_bit_value(options, shape):
    """One key: the output is its value, every e4m3 there is, exactly (powers of two as scales); NaN stays NaN."""
    options("paged_shape", shape)
    c = Case([1], 1, 2, 2, 128, 16, e4m3=True)
    page = int(c.table[0, 0])
    c.pages[1].view(torch.uint8)[page, :, 0] = torch.arange(256, dtype=torch.uint8, device=DEV).view(2, 128)
    c.scales[1].copy_(torch.tensor([0.25, 8.0], device=DEV))
    c.run()
    want = heads.e4m3_values().reshape(2, 128) * np.array([[0.25], [8.0]])
    assert np.array_equal(wide(c.out)[0, 0], want, equal_nan=True)
    # and as a key: the score of a query of ones at one entry
    c.pages[0].view(torch.uint8)[page, 0, 0] = torch.arange(128, dtype=torch.uint8, device=DEV)
    c.pages[0].view(torch.uint8)[page, 0, 0, 127] = 0
    c.q.zero_()
    c.q[0, 0, 0] = 1.0
    c.scales[0].fill_(0.5)
    c.run(scale=1.0)
    assert abs(float(c.lse[0, 0, 0]) - heads.e4m3_values()[:127].sum() * 0.5) <= 1e-5 * heads.e4m3_values()[:127].sum()


def test_scores_far_apart():
    """One key that outweighs all others in a late tile, and scores in the hundreds."""
    c = Case([900], 1, 4, 2, 128, 64)
    c.q *= 30.0
    c.run()
    c.check()
    c.run(scale=1.0)
    c.check(scale=1.0)


def test_views_another_stream_and_repeats():
    c = Case([700, 90], 4, 8, 2, 128, 32)
    c.run()
    first = c.out.clone(), c.lse.clone()
    wide_q, wide_out = torch.zeros((2, 6, 12, 160), dtype=BF16, device=DEV), torch.full((2, 8, 5, 128), 7.0, dtype=BF16, device=DEV)
    q, out = wide_q[:, 1:5, 2:10, 16:144], wide_out.permute(0, 2, 1, 3)[:, 1:]          # [B, Lq, Hq, d], heads outside
    q.copy_(c.q)
    ws = torch.empty(dlm.paged_attn_workspace_bytes(q, out, *c.pages, c.table, c.lens), dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            dlm.paged_attn(q, out, *c.pages, c.table, c.lens, lse=c.lse, workspace=ws)
    dlm.paged_attn(c.q, c.out, *c.pages, c.table, c.lens, stream=side, workspace=ws)
    torch.cuda.synchronize()
    assert torch.equal(out, first[0]) and torch.equal(c.out, first[0]) and torch.equal(c.lse, first[1])
    assert (wide_out.permute(0, 2, 1, 3)[:, :1] == 7).all()


def test_pages_past_32_bits_of_offset():
    """Pages 2^31 entries apart."""
    d, page, far = 64, 16, 1 << 31
    c = Case([40], 1, 2, 1, d, page, spare=0)
    flat = torch.zeros(2 * far + 2 * page * d, dtype=BF16, device=DEV)
    pages = [flat.as_strided((3, 1, page, d), (far, page * d, d, 1), i * page * d) for i in range(2)]
    for new, old in zip(pages, c.pages):
        new.copy_(old)
    c.pages = pages
    c.run()
    c.check()


@pytest.mark.parametrize("bs", [0, 1, 32])
def test_whole_prompts(bs):
    """As many queries as keys, and more or fewer of them: many row groups a sequence, the later ones with more keys."""
    mask = dict(mask_mode=dlm.MASK_BLOCK_CAUSAL, block_size=bs) if bs else {}
    for Hq, Hkv, d, e4m3 in ((7, 1, 64, False), (2, 1, 128, False), (2, 2, 128, True)):
        c = Case([401, 90, 400, 800], 400, Hq, Hkv, d, 32, e4m3, q_len=[400, 90, 33, 399])
        c.run(**mask)
        c.check(**mask)


@pytest.mark.parametrize("shape", [0, 2, 3])
def test_pages_that_sequences_share(options, shape):
    """A common beginning in the same pages, a page twice in one sequence, two sequences of the same pages throughout."""
    options("paged_shape", shape)
    c = Case([500, 300, 300, 64], 3, 8, 2, 64, 32)
    t = c.table
    t[1, :5] = t[0, :5]
    t[2] = t[1]
    t[3, 1] = t[3, 0]
    for mask in ({}, dict(mask_mode=dlm.MASK_BLOCK_CAUSAL, block_size=1)):
        c.run(**mask)
        c.check(**mask)


@pytest.mark.parametrize("shape", [2, 3])
def test_two_calls_at_once(options, shape):
    """Two streams, a workspace each: what each gives alone."""
    options("paged_shape", shape)
    options("paged_shares", 300)
    a, b = Case([6000, 100], 4, 8, 2, 64, 64, seed=1), Case([300, 5000, 2000], 8, 4, 4, 128, 16, seed=2)
    want = []
    for c in (a, b):
        assert c.run() > 0
        want.append((c.out.clone(), c.lse.clone()))
    spaces, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for c in (a, b):
        given = (c.q, c.out, *c.pages, c.table, c.lens)
        spaces.append(torch.empty(dlm.paged_attn_workspace_bytes(*given, lse=c.lse), dtype=torch.uint8, device=DEV))
        c.out.zero_(), c.lse.zero_()
    torch.cuda.synchronize()
    for _ in range(5):
        for c, ws, s in zip((a, b), spaces, streams):
            with torch.cuda.stream(s):
                dlm.paged_attn(c.q, c.out, *c.pages, c.table, c.lens, lse=c.lse, workspace=ws)
    torch.cuda.synchronize()
    for c, (out, lse) in zip((a, b), want):
        assert torch.equal(c.out, out) and torch.equal(c.lse, lse)


@pytest.mark.parametrize("shape", [2, 3])
def test_captured_and_replayed(options, shape):
    """Shares in a graph: replays with other lengths, numbers of rows and pages, eager calls in between."""
    options("paged_shape", shape)
    options("paged_shares", 64)
    c = Case([900, 2000, 40], 5, 8, 2, 128, 32, q_len=[5, 5, 5])
    given, how = (c.q, c.out, *c.pages, c.table, c.lens), dict(q_len=c.q_len, lse=c.lse)
    ws = torch.empty(dlm.paged_attn_workspace_bytes(*given, **how), dtype=torch.uint8, device=DEV)
    assert ws.numel() > 0
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dlm.paged_attn(*given, workspace=ws, **how)
    for lens, rows in (([900, 2000, 40], [5, 5, 5]), ([2000, 0, 1], [1, 0, 5]), ([33, 32, 31], [0, 0, 0]), ([1, 2000, 1999], [5, 3, 4])):
        c.lens.copy_(torch.tensor(lens, dtype=I32)), c.q_len.copy_(torch.tensor(rows, dtype=I32))
        c.table.clamp_(min=0)
        c.out.fill_(7.0), c.lse.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        c.lengths = lens
        c.check()
        got = c.out.clone(), c.lse.clone()
        c.out.fill_(7.0), c.lse.fill_(7.0)
        c.run()
        assert torch.equal(c.out, got[0]) and torch.equal(c.lse, got[1])
