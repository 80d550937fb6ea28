"""The LM head's gradient without a GPU: struct layout, what the call refuses before any device work, and its workspace."""
import ctypes as C
import os
import subprocess

import pytest
import torch

import rows_structs as S
from paper_2604_04215_amd import binding as dlm

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BAD, UNSUPPORTED, WORKSPACE = dlm.DLM_ERR_INVALID_ARG, dlm.DLM_ERR_UNSUPPORTED, dlm.DLM_ERR_WORKSPACE
P = 0x10000


def test_struct_layout_matches_header(tmp_path):
    s = S.LmheadBwdArgs
    prog, exe = tmp_path / "layout.c", tmp_path / "layout"
    prog.write_text("#include <stdio.h>\n#include <stddef.h>\n#include \"dlm.h\"\nint main(void) {printf(\"%zu\\n\", sizeof(dlm_lmhead_bwd_args));"
                    + "".join(f'printf("%zu\\n", offsetof(dlm_lmhead_bwd_args, {f[0]}));' for f in s._fields_) + "return 0; }")
    subprocess.check_call(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), str(prog), "-o", str(exe)])
    got = [int(x) for x in subprocess.check_output([str(exe)], text=True).split()]
    assert got == [C.sizeof(s)] + [getattr(s, f[0]).offset for f in s._fields_]


def _args(**kw):
    a = S.LmheadBwdArgs()
    f = dict(struct_size=C.sizeof(a), M=4, Dh=64, V=10, hidden=P, hidden_stride_row=64, w=P, w_stride_row=64, inv_temperature=1.0, forbid_token=-1, lse=P, target=P, d_lse=P,
             d_ztarget=P, d_hidden=P, d_hidden_stride_row=64, d_w=3 * P, d_w_stride_row=64, workspace=P, workspace_bytes=1 << 30)
    for k, v in dict(f, **kw).items():
        setattr(a, k, v)
    return a


REFUSED = [(dict(struct_size=8), BAD), (dict(M=-1), BAD), (dict(Dh=0), BAD), (dict(V=0), BAD), (dict(Dh=72), UNSUPPORTED), (dict(M=(1 << 20) + 1), UNSUPPORTED),
           (dict(Dh=1 << 17), UNSUPPORTED), (dict(V=(1 << 24) + 1), UNSUPPORTED), (dict(forbid_token=10), BAD), (dict(inv_temperature=0.0), BAD),
           (dict(inv_temperature=float("nan")), BAD), (dict(inv_temperature=float("inf")), BAD), (dict(d_hidden=None, d_w=None), BAD),
           (dict(d_lse=None, d_ztarget=None), BAD), (dict(target=None), BAD), (dict(lse=None), BAD), (dict(hidden=None), BAD), (dict(w=None), BAD),
           (dict(hidden=P + 8), UNSUPPORTED), (dict(w=P + 2), UNSUPPORTED), (dict(w_stride_row=32), BAD), (dict(hidden_stride_row=0), BAD), (dict(w_stride_row=68), UNSUPPORTED),
           (dict(w_stride_row=1 << 23), UNSUPPORTED), (dict(d_hidden_type=2), BAD), (dict(d_w_type=-1), BAD), (dict(d_hidden_stride_row=56), BAD), (dict(d_w_stride_row=0), BAD),
           (dict(d_w=P + 8), UNSUPPORTED), (dict(d_w=P), BAD), (dict(d_w=3 * P, d_hidden=3 * P), BAD), (dict(d_w_type=1, d_w_stride_row=66), UNSUPPORTED), (dict(workspace=None), WORKSPACE), (dict(workspace_bytes=100), WORKSPACE),
           (dict(workspace=P + 8), WORKSPACE)]


@pytest.mark.parametrize("fields,code", REFUSED)
def test_refused(fields, code):
    assert dlm.lib().dlm_lmhead_bwd(C.byref(_args(**fields)), None) == code
    assert "lmhead_bwd" in dlm.last_error()


def test_nothing_to_do():
    for kw in (dict(d_w=None), dict(accumulate=1)):
        assert dlm.lib().dlm_lmhead_bwd(C.byref(_args(M=0, hidden=None, lse=None, w=None, workspace=None, d_hidden=None if "accumulate" in kw else P, **kw)), None) == dlm.DLM_OK
    assert dlm.lib().dlm_lmhead_bwd(None, None) == BAD


def test_workspace_sizes():
    size = dlm.lib().dlm_lmhead_bwd_workspace_bytes
    size.restype = C.c_size_t
    assert size(None) == 0 and size(C.byref(_args(struct_size=4))) == 0
    small, big = size(C.byref(_args())), size(C.byref(_args(M=1 << 20, V=1 << 24, Dh=4096)))
    assert 64 * 64 * 4 < small < 1 << 21 and big < 1 << 40
    for M in (1, 65, 512, 4096, 32768):
        kw = dict(M=M, V=126464, Dh=4096, w_stride_row=4096, hidden_stride_row=4096)
        both, rows, weights = (size(C.byref(_args(**kw, **m))) for m in ({}, dict(d_w=None), dict(d_hidden=None)))
        assert weights < both and weights < rows
        most = (2 << 30) + 2 * (M + 63) * 4096 * 2 + 3 * 64 * M * 4096 * 4 + (8 << 20)
        assert both <= most + 126464 * 4096 * 2              # a copy of W
        assert size(C.byref(_args(**kw, d_w_type=1))) <= most and rows <= most + 126464 * 4096 * 2


def test_binding_refuses_what_is_not_on_the_gpu():
    x, f = torch.zeros((4, 64), dtype=torch.bfloat16), torch.zeros(4)
    for call in (lambda: dlm.lmhead_bwd(x, x, f, d_lse=f, d_w=x), lambda: dlm.lmhead_bwd_workspace_bytes(x, x, f, d_lse=f, d_w=x)):
        with pytest.raises(ValueError, match="GPU"):
            call()
