"""Outputs of the norms in the place of their inputs: what is refused before any device work (no GPU)."""
import ctypes as C

import pytest

from paper_2604_04215_amd import binding as dlm
from test_rows_boundary import BAD, P, _norm, _norm_bwd

F32 = 1
Q = 5 * P


@pytest.mark.parametrize("fields,why", [
    (dict(out=Q, sum_out=Q), "the sum would be lost"),
    (dict(x=Q, out=Q, sum_out=Q), "also in the place of x, where each may be by itself"),
    (dict(x=Q, out=Q, x_type=F32), "rows of half the size"),
    (dict(x=Q, out=Q, x_stride=128), "other rows"),
    (dict(residual=Q, out=Q, x_type=F32), "rows of half the size"),
    (dict(residual=Q, out=Q, residual_stride=128), "other rows"),
    (dict(x=Q, sum_out=Q, sum_stride=128), "other rows"),
    (dict(residual=Q, sum_out=Q, sum_stride=72), "other rows")])
def test_norm(fields, why):
    free = dict(x=P, residual=2 * P, sum_out=3 * P, out=4 * P)
    assert dlm.lib().dlm_row_norm(C.byref(_norm(**dict(free, **fields))), None) == BAD, why
    assert "row_norm" in dlm.last_error()


@pytest.mark.parametrize("fields,why", [
    (dict(x=Q, d_x=Q, d_x_stride=128), "other rows"),
    (dict(d_sum=Q, d_x=Q, d_sum_stride=128), "other rows"),
    (dict(d_out=Q, d_x=Q, d_out_stride=128), "other rows"),
    (dict(d_out=Q, d_x=Q, x_type=F32), "rows of twice the size")])
def test_norm_gradient(fields, why):
    free = dict(d_out=P, x=2 * P, d_sum=3 * P, d_x=4 * P)
    assert dlm.lib().dlm_row_norm_bwd(C.byref(_norm_bwd(**dict(free, **fields))), None) == BAD, why
    assert "row_norm_bwd" in dlm.last_error()
