"""The residual-block operators without rows: matrices and vectors of rows have no element and may be NULL, as an empty
tensor's address is.  Host checks only; nothing here launches a kernel."""
import pytest

import paper_1811_12843_amd as L

from test_abi_blocks import NONE, linear, linear_bwd, linear_fp8, norm, norm_bwd

EMPTY = L.lipz_mat(None, 40, 40)  # an empty tensor's strides

CASES = [
    (norm, "lipz_rms_norm", dict(x=EMPTY, residual=EMPTY, h=EMPTY, y=EMPTY, rstd=None, y_scale=None)),
    (norm, "lipz_rms_norm", dict(x=EMPTY, residual=EMPTY, h=EMPTY, y=EMPTY, rstd=None, y_scale=None, y_dtype=L.LIPZ_FP8)),
    (norm_bwd, "lipz_rms_norm_backward", dict(h=EMPTY, dy=EMPTY, dh=EMPTY, dx=EMPTY, rstd=None, dgamma=None)),
    (linear, "lipz_linear", dict(x=EMPTY, residual=EMPTY, pre=EMPTY, y=EMPTY)),
    (linear_fp8, "lipz_linear_fp8", dict(x=EMPTY, residual=EMPTY, y=EMPTY, x_scale=None)),
]


@pytest.mark.parametrize("make,name,kw", CASES)
def test_calls_without_rows_take_null(make, name, kw):
    a = make(rows=0, **kw)
    nb = getattr(L, name + "_workspace_bytes")(a)
    assert nb > 0
    getattr(L, name)(a, 1 << 20, nb, None)  # nothing to do
    assert getattr(L, name + "_workspace_bytes")(make(rows=1, **kw)) == 0


@pytest.mark.parametrize("kw", [dict(), dict(dw=NONE), dict(db=None), dict(dw=NONE, db=None), dict(w=NONE)])
def test_gradients_without_rows_take_null(kw):
    empty = dict(x=EMPTY, pre=EMPTY, dy=EMPTY, dx=EMPTY)
    need = L.lipz_linear_backward_workspace_bytes
    assert need(linear_bwd(rows=0, **empty, **kw)) > 0 and need(linear_bwd(rows=1, **empty, **kw)) == 0


def test_what_does_not_depend_on_rows_is_still_checked():
    need = L.lipz_rms_norm_workspace_bytes, L.lipz_linear_workspace_bytes, L.lipz_linear_fp8_workspace_bytes
    assert need[0](norm(rows=0, gamma=None)) == need[1](linear(rows=0, w=NONE)) == need[2](linear_fp8(rows=0, w=NONE)) == 0
    assert L.lipz_linear_backward_workspace_bytes(linear_bwd(rows=0, w=NONE)) == 0  # dx has an address
    assert need[2](linear_fp8(rows=0, w_scale=None)) == 0
