"""Limits of the residual-block operators apply to what a call asks for.  Host checks only."""
import pytest

import paper_1811_12843_amd as L

from test_abi_blocks import NONE, linear_bwd


@pytest.mark.parametrize("left_out", ["dx", "dw"])
def test_a_gradient_left_out_has_no_size_limit(left_out):
    """Many cells that share their weights: dw per cell would pass the limit on blocks of outputs, dx does not; and with
    many rows and few outputs dx would."""
    C, (M, K, N) = 65535, {"dw": (1, 1040, 1040), "dx": (1040, 1040, 1)}[left_out]
    kw = dict(cells=C, rows=M, fan_in=K, fan_out=N, act=L.LIPZ_ACT_LINEAR, pre=NONE, db=None, x=L.lipz_mat(1 << 20, K, 0),
              w=L.lipz_mat(1 << 20, N, 0), dy=L.lipz_mat(1 << 20, N, M * N), dx=L.lipz_mat(1 << 20, K, M * K),
              dw=L.lipz_mat(1 << 20, N, K * N))
    need = L.lipz_linear_backward_workspace_bytes
    assert need(linear_bwd(**kw)) == 0
    assert need(linear_bwd(**dict(kw, **{left_out: NONE}))) > 0
