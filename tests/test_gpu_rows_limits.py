"""The embedding's gradient at the ends of what it takes (GPU).  Small whole numbers: every sum is exact."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2604_04215_amd import binding as dlm
from gpu_util import DEV

pytestmark = pytest.mark.gpu
F32, I32, U8 = torch.float32, torch.int32, torch.uint8


def test_as_many_entries_as_are_taken():
    """2^40 entries of fp32 (one row for all tokens): the sums' workgroups have 2^32 threads together."""
    T, Dh = 1 << 24, 1 << 16
    row = (torch.arange(Dh, device=DEV) % 3 - 1).float()
    tokens = (torch.arange(T, device=DEV) * 7 % 16).to(I32)
    tokens = torch.where(tokens < 8, 0, torch.where(tokens < 12, 1, torch.where(tokens < 14, 2, -1))).to(I32)
    table = torch.full((3, Dh), 5.0, dtype=F32, device=DEV)
    ws = torch.empty(dlm.embed_bwd_workspace_bytes(T, 3, Dh), dtype=U8, device=DEV)
    dlm.embed_bwd(tokens, row.expand(T, Dh), table, workspace=ws)
    for v, n in enumerate((T // 2, T // 4, T // 8)):
        assert torch.equal(table[v], n * row), v


def launches(call):
    """Launches of a captured call."""
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        call()
    n = C.c_size_t()
    assert dlm.lib().hipGraphGetNodes(C.c_void_p(graph.raw_cuda_graph()), None, C.byref(n)) == 0
    return n.value


@pytest.mark.parametrize("T,accumulate,merges", [(70000, False, 1), (70000, True, 2), (140001, True, 2), (270001, False, 2), (2100001, True, 3), (2100001, False, 2)])
def test_levels_of_merging(T, accumulate, merges):
    """Up to 32 runs are merged at once: of 2048 tokens where sums are added (35, 69 and 1026 runs here), of 8192 where a table is cleared (9, 33, 257).  Exact, every time."""
    V, Dh, rng = 3000, 8, np.random.default_rng(T)
    at = np.arange(T)
    tokens = np.where(rng.random(T) < 0.4, V - 1, rng.integers(-3, V + 3, T)).astype(np.int32)
    dy = (at[:, None] * 7 + np.arange(Dh)) % 13 - 6
    want = np.zeros((V, Dh))
    live = (tokens >= 0) & (tokens < V)
    np.add.at(want, tokens[live], dy[live])
    d_out, dev = torch.from_numpy(dy).to(torch.bfloat16).to(DEV), torch.from_numpy(tokens).to(DEV)
    ws = torch.empty(dlm.embed_bwd_workspace_bytes(T, V, Dh), dtype=U8, device=DEV)
    table = torch.empty((V, Dh), dtype=F32, device=DEV)
    call = lambda: dlm.embed_bwd(dev, d_out, table, accumulate=accumulate, workspace=ws)
    assert launches(call) == 3 + merges                 # sort, merges, sums, join
    for fill in (3.0, -5.0):
        table.fill_(fill)
        ws.fill_(255)
        call()
        assert np.array_equal(table.double().cpu().numpy(), want + (fill if accumulate else 0))


def test_gradients_on_two_streams_at_once():
    """Neither waits for the other: each has its own workspaces."""
    rng = np.random.default_rng(1)
    T, V, D = 20000, 900, 520
    tokens = torch.from_numpy(rng.integers(-1, V, T).astype(np.int32)).to(DEV)
    x, dy = (torch.from_numpy(rng.standard_normal((T, D)).astype(np.float32)).to(torch.bfloat16).to(DEV) for _ in range(2))
    runs = [dict(table=torch.zeros((V, D), dtype=F32, device=DEV), d_x=torch.zeros_like(x), d_w=torch.zeros(D, device=DEV), d_b=torch.zeros(D, device=DEV),
                 ws=[torch.empty(n, dtype=U8, device=DEV) for n in (dlm.row_norm_bwd_workspace_bytes(T, D), dlm.embed_bwd_workspace_bytes(T, V, D))]) for _ in range(3)]

    def chain(r, **kw):
        dlm.row_norm_bwd(dy, x, r["d_x"], kind=dlm.NORM_LAYER, d_weight=r["d_w"], d_bias=r["d_b"], workspace=r["ws"][0], **kw)
        dlm.embed_bwd(tokens, r["d_x"], r["table"], workspace=r["ws"][1], **kw)

    chain(runs[2])
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(8):
        for s, r in zip(streams, runs):
            chain(r, stream=s)
    torch.cuda.synchronize()
    for r in runs[:2]:
        assert all(torch.equal(r[k], runs[2][k]) for k in ("table", "d_x", "d_w", "d_b"))


@pytest.mark.parametrize("T,D", [(5, 72), (33, 1032), (2100, 4096)])
def test_norm_in_the_place_of_the_residual(T, D):
    rng = np.random.default_rng(T)
    x, residual = (torch.from_numpy(rng.standard_normal((T, D)).astype(np.float32)).to(torch.bfloat16).to(DEV) for _ in range(2))
    total, out, total2 = (torch.zeros_like(x) for _ in range(3))
    dlm.row_norm(x, out, residual=residual, sum_out=total, kind=dlm.NORM_LAYER)
    dlm.row_norm(x, residual, residual=residual, sum_out=total2, kind=dlm.NORM_LAYER)
    assert torch.equal(residual, out) and torch.equal(total2, total)
    with pytest.raises(dlm.DlmError):
        dlm.row_norm(x, x, residual=out, sum_out=x)
