"""The workspace of paged attention without a GPU: what is refused, and the bound on its size."""
import ctypes as C
import random

import test_heads_boundary as boundary
from paper_2604_04215_amd import binding as dlm


def size(**kw):
    L = dlm.lib()
    L.dlm_paged_attn_workspace_bytes.restype = C.c_size_t
    return L.dlm_paged_attn_workspace_bytes(C.byref(boundary._attn(**kw)))


def test_misaligned_workspace_is_refused():
    for at in (4, 8, boundary.P + 8):
        for nbytes in (0, 1 << 30):
            assert dlm.lib().dlm_paged_attn(C.byref(boundary._attn(workspace=at, workspace_bytes=nbytes)), None) == dlm.DLM_ERR_WORKSPACE
            assert "not 16-byte aligned" in dlm.last_error()


def test_size_is_bounded_whatever_the_call():
    """Its documented bound, over batches, lengths, heads and masks; and that it does rise where a batch gets smaller."""
    rng, seen = random.Random(3), 0
    for _ in range(20000):
        Hkv, g, d = rng.choice([1, 2, 4, 8, 32]), rng.choice([1, 4, 7, 8, 16]), rng.choice([64, 128])
        B, Lq, n = int(2 ** rng.uniform(0, 10)), int(2 ** rng.uniform(0, 13)), int(2 ** rng.uniform(0, 20))
        got = size(B=B, Lq=Lq, Hq=g * Hkv, Hkv=Hkv, d=d, max_kv_len=n, table_stride=1 << 20, mask_mode=rng.choice([0, 1]), block_size=rng.choice([1, 32]),
                   cache=boundary._cache(type=rng.choice([0, 1])))
        assert got <= 2 ** 18 * (d + 2) + 8 * B * Hkv * -(-Lq * g // 32)
        seen += got > 0
    assert seen > 2000
    few, many = (size(B=B, Hq=32, Hkv=8, max_kv_len=4096, table_stride=1 << 20) for B in (8, 64))
    assert few > 0 and many == 0
