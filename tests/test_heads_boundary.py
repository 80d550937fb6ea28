"""Paged cache, head norms and rotation without a GPU: struct layout, and what the calls refuse before any device work."""
import ctypes as C
import os
import subprocess

import pytest
import torch

import heads_structs as S
from paper_2604_04215_amd import binding as dlm

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STRUCTS = [("dlm_paged_kv", S.PagedKv), ("dlm_head_map", S.HeadMap), ("dlm_qk_args", S.QkArgs), ("dlm_qk_bwd_args", S.QkBwdArgs),
           ("dlm_append_args", S.AppendArgs), ("dlm_paged_attn_args", S.PagedAttnArgs)]
BAD, UNSUPPORTED, WORKSPACE = dlm.DLM_ERR_INVALID_ARG, dlm.DLM_ERR_UNSUPPORTED, dlm.DLM_ERR_WORKSPACE


def test_struct_layout_matches_header(tmp_path):
    lines = [f'printf("%zu\\n", sizeof({n}));' + "".join(f'printf("%zu\\n", offsetof({n}, {f[0]}));' for f in s._fields_) for n, s in STRUCTS]
    prog, exe = tmp_path / "layout.c", tmp_path / "layout"
    prog.write_text("#include <stdio.h>\n#include <stddef.h>\n#include \"dlm.h\"\nint main(void) {" + "\n".join(lines) + "return 0; }")
    subprocess.check_call(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), str(prog), "-o", str(exe)])
    got = [int(x) for x in subprocess.check_output([str(exe)], text=True).split()]
    want = [x for _, s in STRUCTS for x in [C.sizeof(s)] + [getattr(s, f[0]).offset for f in s._fields_]]
    assert got == want


P = 0x10000


def _map(**kw):
    return dict(dict(q_weight=P, k_weight=P, eps=1e-6, rope=P, rope_len=64, rot_dim=128, rope_style=0, positions=P), **kw)


def _fill(struct, fields):
    for k, v in fields.items():
        if isinstance(v, dict):
            _fill(getattr(struct, k), v)
        else:
            setattr(struct, k, v)
    return struct


def _qk(**kw):
    f = dict(struct_size=C.sizeof(S.QkArgs), T=4, Hq=4, Hkv=2, d=128, q=P, k=P, q_out=P, k_out=P, map=_map())
    for x, h in (("q", 4), ("k", 2), ("qo", 4), ("ko", 2)):
        f[x + "_stride_t"], f[x + "_stride_h"] = h * 128, 128
    return _fill(S.QkArgs(), dict(f, **kw))


def _bwd(**kw):
    f = dict(struct_size=C.sizeof(S.QkBwdArgs), T=4, Hq=4, Hkv=2, d=128, d_q_out=P, d_k_out=P, q=P, k=P, d_q=P, d_k=P, d_q_weight=P, d_k_weight=P,
             map=_map(), workspace=P, workspace_bytes=1 << 20)
    for x, h in (("dqo", 4), ("dko", 2), ("q", 4), ("k", 2), ("dq", 4), ("dk", 2)):
        f[x + "_stride_t"], f[x + "_stride_h"] = h * 128, 128
    return _fill(S.QkBwdArgs(), dict(f, **kw))


def _cache(**kw):
    return dict(dict(k=P, v=P, n_pages=8, page_size=16, stride_page=2 * 16 * 128, stride_h=16 * 128, stride_t=128, type=0), **kw)


def _append(**kw):
    f = dict(struct_size=C.sizeof(S.AppendArgs), T=4, Hq=4, Hkv=2, d=128, q=P, k=P, v=P, q_out=P, slots=P, cache=_cache(), map=_map())
    for x, h in (("q", 4), ("k", 2), ("v", 2), ("qo", 4)):
        f[x + "_stride_t"], f[x + "_stride_h"] = h * 128, 128
    return _fill(S.AppendArgs(), dict(f, **kw))


def _attn(**kw):
    f = dict(struct_size=C.sizeof(S.PagedAttnArgs), B=2, Lq=1, Hq=4, Hkv=2, d=128, q=P, out=P, cache=_cache(), block_table=P, table_stride=4, kv_len=P,
             max_kv_len=64)
    for x in "qo":
        f[x + "_stride_b"], f[x + "_stride_t"], f[x + "_stride_h"] = 4 * 128, 4 * 128, 128
    return _fill(S.PagedAttnArgs(), dict(f, **kw))


# rotation and norm: the same for all three calls that have them
MAP = [(dict(eps=-1.0), BAD), (dict(eps=0.0), BAD), (dict(eps=float("nan")), BAD), (dict(rope_style=2), BAD), (dict(rot_dim=8), UNSUPPORTED), (dict(rot_dim=24), UNSUPPORTED),
       (dict(rot_dim=144), UNSUPPORTED), (dict(rope_len=0), BAD), (dict(positions=None), BAD), (dict(rope=P + 4), UNSUPPORTED), (dict(q_weight=P + 2), UNSUPPORTED)]
CACHE = [(dict(type=2), BAD), (dict(n_pages=-1), BAD), (dict(page_size=24), BAD), (dict(page_size=0), BAD), (dict(page_size=8), UNSUPPORTED),
         (dict(page_size=1 << 17), UNSUPPORTED), (dict(n_pages=1 << 27), UNSUPPORTED), (dict(k=None), BAD), (dict(v=P + 8), UNSUPPORTED),
         (dict(stride_t=132), UNSUPPORTED), (dict(stride_page=-4096), UNSUPPORTED), (dict(k_scale=P), BAD), (dict(type=1, stride_t=136), UNSUPPORTED)]
REFUSED = (
    [("dlm_qk_norm_rope", _qk, dict(map=_map(**m)), code) for m, code in MAP]
    + [("dlm_qk_norm_rope_bwd", _bwd, dict(map=_map(**m)), code) for m, code in MAP]
    + [("dlm_paged_append", _append, dict(map=_map(**m)), code) for m, code in MAP]
    + [("dlm_paged_append", _append, dict(cache=_cache(**c)), code) for c, code in CACHE]
    + [("dlm_paged_attn", _attn, dict(cache=_cache(**c)), code) for c, code in CACHE]
    + [("dlm_qk_norm_rope", _qk, kw, code) for kw, code in [
        (dict(struct_size=8), BAD), (dict(T=-1), BAD), (dict(d=96), UNSUPPORTED), (dict(q=None), BAD), (dict(q=P + 4), UNSUPPORTED), (dict(k_out=None), BAD),
        (dict(q_stride_t=516), UNSUPPORTED), (dict(qo_stride_t=256), BAD), (dict(qo_stride_h=64), BAD), (dict(ko_stride_t=0), BAD), (dict(T=1 << 30), UNSUPPORTED), (dict(T=1 << 28), UNSUPPORTED)]]
    + [("dlm_qk_norm_rope_bwd", _bwd, kw, code) for kw, code in [
        (dict(struct_size=8), BAD), (dict(d_q_out=None), BAD), (dict(q=None), BAD), (dict(d_k=P + 2), UNSUPPORTED), (dict(dk_stride_t=128), BAD),
        (dict(map=_map(q_weight=None)), BAD), (dict(workspace=None), WORKSPACE), (dict(workspace_bytes=16), WORKSPACE), (dict(workspace=P + 4), WORKSPACE)]]
    + [("dlm_paged_append", _append, kw, code) for kw, code in [
        (dict(struct_size=8), BAD), (dict(Hkv=0), BAD), (dict(v=None), BAD), (dict(slots=None), BAD), (dict(q_out=None), BAD), (dict(v_stride_h=100), UNSUPPORTED),
        (dict(cache=_cache(stride_h=128)), BAD), (dict(cache=_cache(stride_page=2048)), BAD), (dict(T=1 << 28), UNSUPPORTED)]]
    + [("dlm_paged_attn", _attn, kw, code) for kw, code in [
        (dict(struct_size=8), BAD), (dict(Hkv=3), BAD), (dict(Hkv=0), BAD), (dict(d=256), UNSUPPORTED), (dict(mask_mode=2), BAD), (dict(mask_mode=1), BAD),
        (dict(scale=float("nan")), BAD), (dict(max_kv_len=-1), BAD), (dict(max_kv_len=65), BAD), (dict(table_stride=-1), BAD), (dict(q=None), BAD),
        (dict(kv_len=None), BAD), (dict(block_table=None), BAD), (dict(out=P + 8), UNSUPPORTED), (dict(q_stride_b=516), UNSUPPORTED), (dict(o_stride_h=64), BAD),
        (dict(o_stride_b=128), BAD), (dict(Lq=1 << 30, Hq=8), UNSUPPORTED),
        (dict(B=1, Lq=1 << 28, Hkv=1), UNSUPPORTED)]])


@pytest.mark.parametrize("name,make,fields,code", REFUSED)
def test_refused_before_any_device_work(name, make, fields, code):
    assert getattr(dlm.lib(), name)(C.byref(make(**fields)), None) == code
    assert name[4:] in dlm.last_error()


def test_null_args_and_empty_problems():
    L = dlm.lib()
    for name in ("dlm_qk_norm_rope", "dlm_qk_norm_rope_bwd", "dlm_paged_append", "dlm_paged_attn"):
        assert getattr(L, name)(None, None) == BAD
    assert L.dlm_qk_norm_rope(C.byref(_qk(T=0, q=None)), None) == dlm.DLM_OK
    assert L.dlm_qk_norm_rope(C.byref(_qk(Hq=0, Hkv=0)), None) == dlm.DLM_OK
    assert L.dlm_qk_norm_rope_bwd(C.byref(_bwd(T=0, d_q_weight=None, d_k_weight=None, workspace=None)), None) == dlm.DLM_OK
    assert L.dlm_paged_append(C.byref(_append(T=0, slots=None)), None) == dlm.DLM_OK
    assert L.dlm_paged_attn(C.byref(_attn(B=0)), None) == dlm.DLM_OK
    assert L.dlm_paged_attn(C.byref(_attn(Lq=0)), None) == dlm.DLM_OK


def test_workspace_sizes():
    assert dlm.qk_norm_rope_bwd_workspace_bytes(0, 4, 2, 128) == 0
    assert dlm.qk_norm_rope_bwd_workspace_bytes(1, 4, 2, 128) == 2 * 128 * 4                    # one workgroup a tensor
    assert 0 < dlm.qk_norm_rope_bwd_workspace_bytes(1 << 20, 32, 8, 64) <= 16386 * 64 * 4        # however many tokens
    L = dlm.lib()
    L.dlm_paged_attn_workspace_bytes.restype = C.c_size_t
    assert L.dlm_paged_attn_workspace_bytes(C.byref(_attn())) == 0                              # four tiles: nothing to share out
    many = L.dlm_paged_attn_workspace_bytes(C.byref(_attn(table_stride=1 << 20, max_kv_len=65536)))
    assert 0 < many < 64 << 20
    assert L.dlm_paged_attn_workspace_bytes(None) == 0


def test_options():
    L = dlm.lib()
    for name, good, bad in (("paged_shape", (1, 2, 3, 4, 0), (-1, 5)), ("paged_shares", (-1, 1, 65536, 0), (-2, 65537))):
        for v in good:
            assert L.dlm_set_option(name.encode(), v) == dlm.DLM_OK
        for v in bad:
            assert L.dlm_set_option(name.encode(), v) == BAD and name in dlm.last_error()


def test_shares_give_every_tile_one_owner():
    """The arithmetic by which workgroups share out the tiles of a batch (sizes, pieces, slots of sums, counts to be joined), over random batches."""
    import random
    rng = random.Random(5)
    for _ in range(3000):
        B, H, shares = rng.randint(1, 9), rng.randint(1, 4), rng.choice([1, 2, 3, 7, 64, 512, 1000])
        tiles = [rng.choice([0, 0, 1, 2, rng.randint(1, 70)]) for _ in range(B)]                # of each row group of a sequence
        groups = [H * rng.randint(1, 3) for _ in range(B)]
        total = sum(t * g for t, g in zip(tiles, groups))
        if total == 0:
            continue
        size = max((total - 1) // shares + 1, 8)
        owned, joined, sums = [0] * total, {}, {}
        for w in range(shares):
            if w * size >= total:
                continue
            at, end, b, base, used = w * size, min(total, (w + 1) * size), 0, 0, set()
            while at < end:
                while at >= base + tiles[b] * groups[b]:
                    base += tiles[b] * groups[b]
                    b += 1
                first = base + (at - base) // tiles[b] * tiles[b]
                stop = min(end, first + tiles[b])
                owned[at:stop] = [n + 1 for n in owned[at:stop]]
                if at == first:
                    joined[first] = (w, (first + tiles[b] - 1) // size - w + 1)
                if not (at == first and stop == first + tiles[b]):
                    slot = 2 * w + (at == first)
                    assert slot not in used and slot < 2 * shares
                    used.add(slot)
                    sums.setdefault(first, []).append(slot)
                at = stop
        assert owned == [1] * total
        for first, (w, n) in joined.items():
            assert sums.get(first, []) == ([2 * (w + s) + (s == 0) for s in range(n)] if n > 1 else [])


def test_binding_refuses_what_is_not_on_the_gpu():
    x = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    for call in (lambda: dlm.qk_norm_rope(x, None, x, None), lambda: dlm.qk_norm_rope_bwd(x, None, x, None), lambda: dlm.paged_append(x, x, x, x, x),
                 lambda: dlm.paged_attn(x, x, x, x, x, x), lambda: dlm.paged_attn_workspace_bytes(x[None], x[None], x[None], x[None], x, x)):
        with pytest.raises(ValueError, match="GPU"):
            call()
    for call in (lambda: dlm.qk_norm_rope(None, None, None, None), lambda: dlm.qk_norm_rope_bwd(None, None, None, None), lambda: dlm.paged_append(None, x, x, x, x)):
        with pytest.raises(ValueError, match="needed"):
            call()
