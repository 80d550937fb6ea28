"""Embedding and norms between layers without a GPU: struct layout, and what the calls refuse before any device work."""
import ctypes as C
import os
import subprocess

import pytest
import torch

import rows_structs as S
from paper_2604_04215_amd import binding as dlm

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STRUCTS = [("dlm_embed_args", S.EmbedArgs), ("dlm_embed_bwd_args", S.EmbedBwdArgs), ("dlm_row_norm_args", S.RowNormArgs),
           ("dlm_row_norm_bwd_args", S.RowNormBwdArgs)]
BAD, UNSUPPORTED, WORKSPACE = dlm.DLM_ERR_INVALID_ARG, dlm.DLM_ERR_UNSUPPORTED, dlm.DLM_ERR_WORKSPACE
P = 0x10000


def test_struct_layout_matches_header(tmp_path):
    lines = [f'printf("%zu\\n", sizeof({n}));' + "".join(f'printf("%zu\\n", offsetof({n}, {f[0]}));' for f in s._fields_) for n, s in STRUCTS]
    prog, exe = tmp_path / "layout.c", tmp_path / "layout"
    prog.write_text("#include <stdio.h>\n#include <stddef.h>\n#include \"dlm.h\"\nint main(void) {" + "\n".join(lines) + "return 0; }")
    subprocess.check_call(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), str(prog), "-o", str(exe)])
    got = [int(x) for x in subprocess.check_output([str(exe)], text=True).split()]
    assert got == [x for _, s in STRUCTS for x in [C.sizeof(s)] + [getattr(s, f[0]).offset for f in s._fields_]]


def _fill(struct, fields, more):
    s = struct()
    for k, v in dict(dict(struct_size=C.sizeof(struct)), **dict(fields, **more)).items():
        setattr(s, k, v)
    return s


def _embed(**kw):
    return _fill(S.EmbedArgs, dict(T=4, V=10, Dh=64, tokens=P, table=P, table_stride=64, scale=1.0, out=P, out_stride=64), kw)


def _embed_bwd(**kw):
    return _fill(S.EmbedBwdArgs, dict(T=4, V=10, Dh=64, tokens=P, d_out=P, d_out_stride=64, scale=1.0, d_table=3 * P, d_table_stride=64, workspace=P,
                                      workspace_bytes=1 << 20), kw)


def _norm(**kw):
    return _fill(S.RowNormArgs, dict(T=4, D=64, x=P, x_stride=64, residual=P, residual_stride=64, sum_out=P, sum_stride=64, weight=P, bias=P, eps=1e-6, out=P,
                                     out_stride=64), kw)


def _norm_bwd(**kw):
    return _fill(S.RowNormBwdArgs, dict(T=4, D=64, d_out=P, d_out_stride=64, x=P, x_stride=64, d_sum=P, d_sum_stride=64, weight=P, eps=1e-6, d_x=P, d_x_stride=64,
                                        d_weight=P, d_bias=P + 512, workspace=P, workspace_bytes=1 << 20), kw)


NAN, INF = float("nan"), float("inf")
TOKENS = [(dict(struct_size=8), BAD), (dict(T=-1), BAD), (dict(V=0), BAD), (dict(Dh=0), BAD), (dict(Dh=60), UNSUPPORTED), (dict(tokens=None), BAD),
          (dict(scale=NAN), BAD), (dict(scale=INF), BAD)]
EPS = [(dict(struct_size=8), BAD), (dict(T=-1), BAD), (dict(D=0), BAD), (dict(D=60), UNSUPPORTED), (dict(D=16392), UNSUPPORTED), (dict(kind=2), BAD), (dict(eps=0.0), BAD),
       (dict(eps=-1.0), BAD), (dict(eps=NAN), BAD), (dict(eps=INF), BAD), (dict(x_type=2), BAD), (dict(x=None), BAD), (dict(x=P + 8), UNSUPPORTED),
       (dict(x_stride=68), UNSUPPORTED), (dict(x_stride=-64), UNSUPPORTED), (dict(x_type=1, x_stride=66), UNSUPPORTED), (dict(weight=P + 2), UNSUPPORTED)]
REFUSED = (
    [("dlm_embed", _embed, kw, code) for kw, code in TOKENS + [
        (dict(out_type=2), BAD), (dict(table=None), BAD), (dict(out=None), BAD), (dict(table=P + 4), UNSUPPORTED), (dict(out_stride=56), BAD),
        (dict(out_stride=68), UNSUPPORTED), (dict(table_stride=-64), UNSUPPORTED)]]
    + [("dlm_embed_bwd", _embed_bwd, kw, code) for kw, code in TOKENS + [
        (dict(d_out_type=3), BAD), (dict(d_table_type=-1), BAD), (dict(V=1 << 21), UNSUPPORTED), (dict(T=(1 << 28) + 1), UNSUPPORTED), (dict(d_out=None), BAD), (dict(d_table=P), BAD),
        (dict(Dh=65544, d_out_stride=65544, d_table_stride=65544), UNSUPPORTED), (dict(T=1 << 28, Dh=8192, d_out_stride=0, d_table_stride=8192), UNSUPPORTED),
        (dict(d_table=None), BAD), (dict(d_table_stride=32), BAD), (dict(d_out_stride=60), UNSUPPORTED), (dict(workspace=None), WORKSPACE),
        (dict(workspace_bytes=16), WORKSPACE), (dict(workspace=P + 4), WORKSPACE)]]
    + [("dlm_row_norm", _norm, kw, code) for kw, code in EPS + [
        (dict(residual=None), BAD), (dict(out=None), BAD), (dict(sum_stride=56), BAD), (dict(residual_stride=4), UNSUPPORTED), (dict(out=P + 2), UNSUPPORTED),
        (dict(bias=P + 4), UNSUPPORTED), (dict(out_stride=32), BAD)]]
    + [("dlm_row_norm_bwd", _norm_bwd, kw, code) for kw, code in EPS + [
        (dict(d_out=None), BAD), (dict(d_x=None), BAD), (dict(d_x_stride=0), BAD), (dict(d_sum=P + 8), UNSUPPORTED), (dict(d_weight=P + 4), UNSUPPORTED),
        (dict(d_bias=P), BAD), (dict(workspace=None), WORKSPACE), (dict(workspace_bytes=64), WORKSPACE), (dict(workspace=P + 8), WORKSPACE)]])


@pytest.mark.parametrize("name,make,fields,code", REFUSED)
def test_refused(name, make, fields, code):
    a = make(**fields)
    assert getattr(dlm.lib(), name)(C.byref(a), None) == code
    assert name[4:] in dlm.last_error()


def test_nothing_to_do_and_null_arguments():
    for name, a in (("dlm_embed", _embed(T=0, tokens=None, out=None)), ("dlm_embed_bwd", _embed_bwd(T=0, tokens=None, d_out=None, accumulate=1, workspace=None)),
                    ("dlm_row_norm", _norm(T=0, x=None, out=None, sum_out=None, residual=None)),
                    ("dlm_row_norm_bwd", _norm_bwd(T=0, x=None, d_out=None, d_x=None, d_sum=None, d_weight=None, d_bias=None, workspace=None))):
        assert getattr(dlm.lib(), name)(C.byref(a), None) == dlm.DLM_OK, dlm.last_error()
        assert getattr(dlm.lib(), name)(None, None) == BAD


def test_workspace_sizes():
    L = dlm.lib()
    L.dlm_embed_bwd_workspace_bytes.restype = L.dlm_row_norm_bwd_workspace_bytes.restype = C.c_size_t
    assert L.dlm_embed_bwd_workspace_bytes(C.byref(_embed_bwd(T=0))) == 0 and L.dlm_row_norm_bwd_workspace_bytes(C.byref(_norm_bwd(T=0))) == 0
    assert L.dlm_embed_bwd_workspace_bytes(None) == 0 and L.dlm_row_norm_bwd_workspace_bytes(C.byref(_norm_bwd(struct_size=1))) == 0
    for T in (1, 333, 2048, 2049, 65536, 1 << 20, 1 << 28):
        n = L.dlm_embed_bwd_workspace_bytes(C.byref(_embed_bwd(T=T, Dh=4096)))
        assert 8 * T <= n <= 16 * T + 64 + 2 * 4 * 4096 * (T // 128 + 1)
    assert L.dlm_row_norm_bwd_workspace_bytes(C.byref(_norm_bwd(T=1 << 30, D=16384))) <= 1 << 27


def test_binding_refuses_what_does_not_fit():
    x, t = torch.zeros((4, 64), dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
    for call in (lambda: dlm.embed(t, x, x), lambda: dlm.embed_bwd(t, x, x), lambda: dlm.row_norm(x, x), lambda: dlm.row_norm_bwd(x, x, x)):
        with pytest.raises(ValueError, match="GPU"):
            call()
