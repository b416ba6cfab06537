"""The residual-block operators on a GPU: empty tensors, and outputs that take the place of inputs."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_1811_12843_amd as L  # noqa: E402

from block_harness import TYPES, blank, call, mat  # noqa: E402


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_empty_tensors(dtype):
    """Gradients of parameters are 0 where the batch is empty, whose tensors have no address."""
    dt, code = TYPES[dtype][:2]
    C, K, N = 2, 24, 13
    x, dx, h, gx = (torch.empty(C, 0, K, device="cuda", dtype=dt) for _ in range(4))
    y, dy, pre = (torch.empty(C, 0, N, device="cuda", dtype=dt) for _ in range(3))
    w, b, gamma = torch.ones(C, K, N, device="cuda", dtype=dt), torch.ones(C, N, device="cuda"), torch.ones(C, K, device="cuda")
    rstd = torch.empty(C, 0, device="cuda")
    assert mat(x).p is None
    dw, ok = blank(C, K, N, dt, 3)
    db, dg = torch.full((C, N), 7.0, device="cuda"), torch.full((C, K), 7.0, device="cuda")
    call("lipz_rms_norm", L.lipz_rms_norm_args(dtype=code, y_dtype=code, cells=C, rows=0, cols=K, eps=1e-5, x=mat(x), y=mat(h),
                                               gamma=gamma.data_ptr(), gamma_cell=K, rstd=rstd.data_ptr()))
    call("lipz_linear", L.lipz_linear_args(dtype=code, cells=C, rows=0, fan_in=K, fan_out=N, act=L.LIPZ_ACT_SILU, slope=0.2,
                                           x=mat(h), w=mat(w), pre=mat(pre), y=mat(y), bias=b.data_ptr(), bias_cell=N))
    call("lipz_linear_backward", L.lipz_linear_backward_args(
        dtype=code, cells=C, rows=0, fan_in=K, fan_out=N, act=L.LIPZ_ACT_SILU, slope=0.2, x=mat(h), w=mat(w), pre=mat(pre),
        dy=mat(dy), dx=mat(dx), dw=mat(dw), db=db.data_ptr(), db_cell=N))
    call("lipz_rms_norm_backward", L.lipz_rms_norm_backward_args(
        dtype=code, cells=C, rows=0, cols=K, h=mat(x), dy=mat(dx), dx=mat(gx), gamma=gamma.data_ptr(), gamma_cell=K,
        rstd=rstd.data_ptr(), dgamma=dg.data_ptr(), dgamma_cell=K))
    assert bool((dw == 0).all()) and bool((db == 0).all()) and bool((dg == 0).all()) and ok()
