"""The embedding's gradient at the ends of what it takes (GPU).  Small whole numbers: every sum is exact."""
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
