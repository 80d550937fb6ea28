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
