"""The LM head's gradient: its workspace, calls beside each other, and what fp32 gradients keep (GPU)."""
import numpy as np
import pytest
import torch

from paper_2604_04215_amd import binding as dlm
from gpu_util import DEV

pytestmark = pytest.mark.gpu
BF16, F32, I32, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


def wide(t):
    return t.detach().double().cpu().numpy()


@pytest.fixture(autouse=True, params=[0, 128], ids=["by itself", "fp16 above 128 rows"])
def few(request):
    """The library's own choice, which for sizes like these is two bf16 terms, and one fp16."""
    dlm.set_option("lmhead_bwd_few", request.param)
    yield
    dlm.set_option("lmhead_bwd_few", 0)


def drawn(M, Dh, V, dtype, seed=0):
    """(hidden, w, lse, the other arguments) of a call"""
    rng = np.random.default_rng(seed + M + V)
    put = lambda x, t: torch.from_numpy(np.ascontiguousarray(x)).to(t).to(DEV)
    h, w = put(rng.standard_normal((M, Dh)), BF16), put(rng.standard_normal((V, Dh)) * 0.3, BF16)
    lse, g = torch.logsumexp(h.float() @ w.float().T, 1), put(rng.standard_normal(M), F32)
    return h, w, lse, dict(target=put(rng.integers(0, V, M), I32), d_ztarget=g, d_lse=-g, d_hidden=torch.zeros((M, Dh), dtype=dtype, device=DEV),
                           d_w=torch.zeros((V, Dh), dtype=dtype, device=DEV))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,V", [(70, 333), (150, 333), (150, 70), (300, 1000), (200, 41000)])
def test_what_is_put_into_the_workspace_does_not_depend_on_what_it_held(M, V, dtype):
    h, w, lse, how = drawn(M, 128, V, dtype)
    held = []
    for fill in (0xaa, 0x55):                            # as exponents of two: below all others, and above
        ws = torch.full((dlm.lmhead_bwd_workspace_bytes(h, w, lse, **how),), fill, dtype=U8, device=DEV)
        dlm.lmhead_bwd(h, w, lse, workspace=ws, **how)
        held.append(ws[2048:])                           # (behind the counters of the tile lists, which end as workgroups come)
    untouched = (held[0] == 0xaa) & (held[1] == 0x55)
    assert ((held[0] == held[1]) | untouched).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,Dh,V", [(300, 1024, 20000), (60, 512, 30000)])
def test_two_calls_at_once(M, Dh, V, dtype):
    """On two streams, neither of which waits for the other: each has its own workspace."""
    h, w, lse, how = drawn(M, Dh, V, dtype)
    size = dlm.lmhead_bwd_workspace_bytes(h, w, lse, **how)
    runs = [dict(how, d_hidden=torch.zeros_like(how["d_hidden"]), d_w=torch.zeros_like(how["d_w"]), workspace=torch.empty(size, dtype=U8, device=DEV)) for _ in range(3)]
    dlm.lmhead_bwd(h, w, lse, **runs[2])
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(4):
        for s, run in zip(streams, runs):
            dlm.lmhead_bwd(h, w, lse, stream=s, **run)
    torch.cuda.synchronize()
    for run in runs[:2]:
        assert torch.equal(run["d_hidden"], runs[2]["d_hidden"]) and torch.equal(run["d_w"], runs[2]["d_w"])


@pytest.mark.parametrize("only", [None, "d_hidden", "d_w"])
@pytest.mark.parametrize("columns", [0, 1024])
def test_16_bit_gradients_of_many_rows_replayed_from_a_graph(columns, only):
    """Other counts, probabilities and workspaces between the replays, with eager calls beside them: the columns' scales are found anew in every call."""
    M, Dh, V = 700, 128, 2600
    h, w, lse, how = drawn(M, Dh, V, BF16)
    idx, count = torch.arange(M, dtype=I32, device=DEV).flip(0).contiguous(), torch.tensor([M], dtype=I32, device=DEV)
    how = dict({k: how[k] for k in ("target", "d_ztarget", "d_lse")}, row_idx=idx, m_dev=count, out_scatter=True, forbid_token=7)
    outs = [{k: t for k, t in (("d_hidden", torch.zeros_like(h)), ("d_w", torch.zeros_like(w))) if only in (None, k)} for _ in range(2)]
    dlm.set_option("lmhead_bwd_columns", columns)
    try:
        ws = [torch.full((dlm.lmhead_bwd_workspace_bytes(h, w, lse, **how, **outs[0]),), 255, dtype=U8, device=DEV) for _ in range(2)]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            dlm.lmhead_bwd(h, w, lse, workspace=ws[1], **how, **outs[1])
        given = lse.clone()
        for live, up in ((700, 0.0), (700, 60.0), (129, 0.0), (0, 0.0), (1, 30.0), (512, 3.0), (700, 0.0)):
            count.fill_(live)
            lse.copy_(given + up * (torch.arange(M, device=DEV) % 3))        # probabilities of every size
            for out, space in zip(outs, ws):
                space.fill_(255)
                for t in out.values():
                    t.fill_(7.0)
            graph.replay()
            dlm.lmhead_bwd(h, w, lse, workspace=ws[0], **how, **outs[0])
            torch.cuda.synchronize()
            for k in outs[0]:
                assert torch.equal(outs[0][k], outs[1][k]) and outs[0][k].isfinite().all(), (live, k)
    finally:
        dlm.set_option("lmhead_bwd_columns", 0)


@pytest.mark.parametrize("M,V", [(200, 1), (200, 33), (129, 64), (1000, 257)])
def test_16_bit_gradients_of_many_rows_added_up(M, V):
    """accumulate: what is added is what is written without it, before its rounding: two roundings of bf16 (2^-8) instead of one."""
    h, w, lse, how = drawn(M, 64, V, BF16)
    base = torch.from_numpy(np.random.default_rng(V).standard_normal((V, 64))).to(BF16).to(DEV)
    ws = torch.empty(dlm.lmhead_bwd_workspace_bytes(h, w, lse, **how), dtype=U8, device=DEV)
    dlm.lmhead_bwd(h, w, lse, workspace=ws, **how)
    alone, added = wide(how["d_w"]), base.clone()
    dlm.lmhead_bwd(h, w, lse, workspace=ws, **dict(how, d_w=added), accumulate=True)
    want = alone + wide(base)
    assert (np.abs(wide(added) - want) <= 2.0 ** -8 * (np.abs(want) + np.abs(alone)) * 1.01 + 2.0 ** -24 * np.abs(wide(base))).all()


# ---- fp32 gradients: sums in two floats, dz of 24 bits ---------------------------------------------------------
# Inputs on which the arithmetic shows: a sum of numbers near one to which, in a later block of the sum, 2^20 and then -2^20 are added.  Added up in one float it
# is rounded to a multiple of 2^-3 (up to 2^-4 off); with each block (128 products of a logit, 256 of a gradient) added to two floats, 2^20 - 2^20 is zero before it meets the rest.
BIG = 2.0 ** 20
U = 2.0 ** -24


def one_float(products):
    """The sum in one float, first to last."""
    x = np.float32(0)
    for p in products.astype(np.float32):
        x = np.float32(x + p)
    return float(x)


def grads(h, w, lse, d_hidden=None, d_w=None, **how):
    put = lambda x, t: torch.from_numpy(np.ascontiguousarray(x)).to(t).to(DEV)
    h, w, lse = put(h, BF16), put(w, BF16), put(lse, F32)
    how = {k: put(v, I32 if k == "target" else F32) for k, v in how.items()}
    out = [torch.full(t.shape, float("nan"), dtype=F32, device=DEV) if on else None for t, on in ((h, d_hidden), (w, d_w))]
    ws = torch.empty(dlm.lmhead_bwd_workspace_bytes(h, w, lse, d_hidden=out[0], d_w=out[1], **how), dtype=U8, device=DEV)
    dlm.lmhead_bwd(h, w, lse, d_hidden=out[0], d_w=out[1], workspace=ws, **how)
    return [None if t is None else wide(t) for t in out]


def rounded(x):
    return wide(torch.from_numpy(x).to(BF16))


@pytest.mark.parametrize("M,V", [(3, 70), (200, 11000)])
def test_logits_of_fp32_gradients_are_sums_in_two_floats(M, V):
    """dz is all of d_w where the hidden row is one in a column of its own; a logit's sum of 128 products is off by at most s(128) of their sizes, 2^-24 2 (16 + 8)."""
    rng = np.random.default_rng(M)
    h, w = np.zeros((M, 256)), np.zeros((V, 256))
    h[:, :128], w[:, :128] = rounded(rng.standard_normal((M, 128)) * 0.3), rounded(rng.standard_normal((V, 128)) * 0.3)
    h[:, [128, 200]], w[:, 128], w[:, 200] = 2.0 ** 10, 2.0 ** 10, -2.0 ** 10
    z, size = h[:, :128] @ w[:, :128].T, np.abs(h[:, :128]) @ np.abs(w[:, :128]).T
    lse = np.float32(np.log(np.exp(z).sum(1)))
    _, d_w = grads(h, w, lse, d_w=True, d_lse=np.eye(M)[0])
    p = np.exp(z[0] - lse[0].astype(np.float64))
    # 2^10 p: three terms of bf16 keep all of p, one product is exact
    err = np.abs(d_w[:, 128] / 2.0 ** 10 / p - 1)
    bound = np.expm1(48 * U * size[0] + 4 * U * (np.abs(z[0]) + abs(lse[0]))) + 16 * U
    assert (err <= bound).all(), (err / bound).max()
    # one float would be far off
    plain = np.array([one_float(h[0] * w[v]) for v in range(20)])
    assert (np.abs(plain - z[0][:20]) > 100 * bound[:20]).mean() > 0.5


def test_large_logits_of_fp32_gradients_keep_what_a_float_cannot_hold():
    """Logits of 4096 + delta, where a float has steps of 2^-11 and delta is less: the difference from lse is formed of both floats."""
    V = 200
    h, w = np.zeros((1, 256)), np.zeros((V, 256))
    h[0, :64], w[:, :64], h[0, 128], w[:, 128] = 8.0, 8.0, 2.0 ** -6, np.arange(V) * 2.0 ** -13
    delta = np.arange(V) * 2.0 ** -19
    _, d_w = grads(h, w, np.float32([4097.0]), d_w=True, d_lse=np.ones(1))
    want = np.exp(delta - 1)
    # the exponent's product by log2(e), the exponential: a few roundings
    assert (np.abs(d_w[:, 0] / 8 / want - 1) <= 16 * U).all(), np.abs(d_w[:, 0] / 8 / want - 1).max() / U
    assert (np.float32(4096 + delta) == 4096).mean() > 0.5 and np.abs(np.exp(-delta) - 1).max() > 1000 * U


@pytest.mark.parametrize("Dh", [128, 5120])
def test_fp32_gradients_of_hidden_rows_are_sums_in_two_floats(Dh):
    """Hidden rows of zeros: all probabilities of a row are exp(-lse)."""
    rng = np.random.default_rng(Dh)
    w = np.zeros((448, Dh))
    w[:256] = rounded(rng.standard_normal((256, Dh)))
    w[300], w[400] = BIG, -BIG
    lse = np.float32(np.log(2.0) * np.array([0, 1, 3, 0.5, 2]))
    d_h, _ = grads(np.zeros((5, Dh)), w, lse, d_hidden=True, d_lse=np.ones(5))
    p, total, size = np.exp(-lse.astype(np.float64))[:, None], w[:256].sum(0), np.abs(w[:256]).sum(0)
    # probabilities 8 u, blocks of 256 products s(256) = 2 u (16 + 16) of their sizes, three terms joined
    bound = p * (np.abs(total) * 8 * U + 64 * U * size + 4 * U * np.abs(total))
    assert (np.abs(d_h - p * total) <= bound).all(), (np.abs(d_h - p * total) / bound).max()
    plain = np.array([one_float(w[:, i]) for i in range(20)])
    assert (np.abs(plain - total[:20]) > 10 * bound[0, :20]).mean() > 0.5


@pytest.mark.parametrize("Dh", [128, 5120])
def test_fp32_gradients_of_w_are_sums_in_two_floats(Dh):
    rng = np.random.default_rng(Dh + 1)
    h, g = np.zeros((448, Dh)), np.zeros(448)
    h[:256], g[:256] = rounded(rng.standard_normal((256, Dh))), np.float32(rng.standard_normal(256))
    h[[300, 400]], g[300], g[400] = 2.0 ** 10, 2.0 ** 10, -2.0 ** 10
    _, d_w = grads(h, np.zeros((448, Dh)), np.zeros(448), d_w=True, d_ztarget=g, target=np.full(448, 7))
    total, size = g[:256] @ h[:256], np.abs(g[:256]) @ np.abs(h[:256])
    # blocks of 256 products of three terms: s(256) of their sizes, and the result's own rounding
    bound = 64 * U * size * 1.01 + U * np.abs(total)
    assert (np.abs(d_w[7] - total) <= bound).all(), (np.abs(d_w[7] - total) / bound).max()
    assert (np.delete(d_w, 7, 0) == 0).all()
    plain = np.array([one_float(g * h[:, i]) for i in range(20)])
    assert (np.abs(plain - total[:20]) > 10 * bound[:20]).mean() > 0.5


@pytest.mark.parametrize("M,Dh,V", [(3, 64, 70), (300, 128, 500), (130, 5120, 400)])
def test_fp32_gradients_keep_24_bits_of_dz(M, Dh, V):
    """One target a row, entries of one: both gradients are dz itself, to the last bit."""
    rng = np.random.default_rng(M)
    g = np.float32(1 + rng.integers(0, 2 ** 23, M) * 2.0 ** -23) * np.float32(2.0) ** rng.integers(-20, 20, M).astype(np.float32)
    d_h, d_w = grads(np.ones((M, Dh)), np.ones((V, Dh)), np.zeros(M), d_hidden=True, d_w=True, d_ztarget=g, target=np.arange(M))
    assert np.array_equal(d_h, np.repeat(g[:, None].astype(np.float64), Dh, 1)) and np.array_equal(d_w[:M], d_h) and (d_w[M:] == 0).all()
    sixteen = lambda x: rounded(x) + rounded(x - rounded(x))        # two terms
    assert (sixteen(g.astype(np.float64)) != g).mean() > 0.9
