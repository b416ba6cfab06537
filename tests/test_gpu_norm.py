"""lipz_rms_norm and lipz_rms_norm_backward against the formulas in 64 bits, through the C ABI.

Tolerances.  fp32 results: sums of n products in any order have a relative error below n 2^-24 in the worst case and
near sqrt(n) 2^-24 in practice; 2e-6 of the row's largest value covers the largest n here.  16-bit results: half a unit
in the last place of the value and the fp32 error below it.  e4m3: half a unit in the last place of the stored value
plus the fp32 error of value and scale (448 at most)."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_1811_12843_amd as L  # noqa: E402

from block_harness import TYPES, blank, call, close, mat, padded  # noqa: E402

DT = ["bf16", "f16", "f32"]
EPS = 1e-5


def norm64(x, r, gamma):
    h = x.double() + (r.double() if r is not None else 0)
    rstd = 1 / torch.sqrt((h * h).mean(2) + EPS)
    return h, rstd, h * rstd[:, :, None] * gamma.double()[:, None]


COLS = [1, 7, 8, 63, 64, 65, 129, 256, 511, 1025, 2048, 2049, 4104, 8191, 16385, 32768, 32769, 70001]


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("cols", COLS)
def test_norm(cols, dtype):
    dt, code = TYPES[dtype][:2]
    g = torch.Generator(device="cuda").manual_seed(cols)
    k = 0
    for cells, rows, res, pad, off in ((1, 1, True, 0, 0), (3, 5, False, 3, 1), (2, 37, True, 8, 0)):
        for fp8 in (False, True):
            k += 1
            print(f"[case] norm {dtype} cols={cols} cells={cells} rows={rows} fp8={fp8}", flush=True)
            x = padded(g, cells, rows, cols, dt, pad, 1.5, off)
            r = padded(g, cells, rows, cols, dt, pad + 1, 0.7, 0) if res else None
            gamma = 1 + 0.1 * torch.randn(cells, cols, generator=g, device="cuda")
            x[0, 0] = 0  # a row of zeros
            if res:
                r[0, 0] = 0
            y, y_ok = blank(cells, rows, cols, torch.float8_e4m3fn if fp8 else dt, 5)
            h, h_ok = blank(cells, rows, cols, dt, 2)
            rstd = torch.full((cells, rows), 7.0, device="cuda")
            scale = torch.full((cells, rows), 7.0, device="cuda")
            call("lipz_rms_norm", L.lipz_rms_norm_args(
                dtype=code, y_dtype=L.LIPZ_FP8 if fp8 else code, cells=cells, rows=rows, cols=cols, eps=EPS, x=mat(x),
                residual=mat(r), h=mat(h) if k % 3 else L.lipz_mat(), y=mat(y), gamma=gamma.data_ptr(), gamma_cell=cols,
                rstd=rstd.data_ptr() if k % 4 else None, y_scale=scale.data_ptr()))
            eh, er, ey = norm64(x, r, gamma)
            if k % 3:
                close(h, eh, dtype, 2.0 ** -24 * eh.abs().amax().item(), "h")
            if k % 4:
                close(rstd, er, "f32", 2e-6 * er, "rstd")
            top = ey.abs().amax(2, keepdim=True)
            if fp8:
                es = torch.clamp_min(ey.abs().amax(2) / 448, 2.0 ** -126)
                close(scale, es, "f32", 4e-6 * es, "scale")
                close(y, ey / es[:, :, None], "fp8", 4e-6 * 448, "y")
            else:
                close(y, ey, dtype, 4e-6 * top, "y")
            assert y_ok() and h_ok()


def test_norm_in_place_and_shared():
    """h may be x or residual; inputs and gamma may be shared between cells."""
    g = torch.Generator(device="cuda").manual_seed(3)
    for cols in (200, 5000, 40000):
        for over in ("x", "residual"):
            x, r = (padded(g, 2, 9, cols, torch.bfloat16, 0) for _ in range(2))
            gamma = 1 + 0.1 * torch.randn(1, cols, generator=g, device="cuda")
            eh, _, ey = norm64(x, r, gamma)
            y, _ = blank(2, 9, cols, torch.bfloat16)
            h = x if over == "x" else r
            call("lipz_rms_norm", L.lipz_rms_norm_args(
                dtype=L.LIPZ_BF16, y_dtype=L.LIPZ_BF16, cells=2, rows=9, cols=cols, eps=EPS, x=mat(x), residual=mat(r),
                h=mat(h), y=mat(y), gamma=gamma.data_ptr(), gamma_cell=0))
            close(h, eh, "bf16", 1e-6, "h")
            close(y, ey, "bf16", 4e-5, "y")
    x = padded(g, 1, 6, 300, torch.float32, 0)
    gamma = 1 + 0.1 * torch.randn(4, 300, generator=g, device="cuda")
    y, _ = blank(4, 6, 300, torch.float32)
    m = mat(x)
    m.cell = 0
    call("lipz_rms_norm", L.lipz_rms_norm_args(dtype=0, y_dtype=0, cells=4, rows=6, cols=300, eps=EPS, x=m, y=mat(y),
                                               gamma=gamma.data_ptr(), gamma_cell=300))
    close(y, norm64(x, None, gamma)[2], "f32", 4e-6 * 6, "y")


@pytest.mark.parametrize("cols", [40, 700, 5000, 40000])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_norm_rows_with_nan_and_infinity(cols, bad):
    """Such a row does not reach its neighbours; in e4m3 its scale and all of it are NaN."""
    g = torch.Generator(device="cuda").manual_seed(4)
    x = padded(g, 1, 11, cols, torch.float32, 1)
    x[0, 4, cols // 2] = bad
    gamma = torch.ones(1, cols, device="cuda")
    y, _ = blank(1, 11, cols, torch.float32)
    call("lipz_rms_norm", L.lipz_rms_norm_args(dtype=0, y_dtype=0, cells=1, rows=11, cols=cols, eps=EPS, x=mat(x),
                                               y=mat(y), gamma=gamma.data_ptr(), gamma_cell=cols))
    close(y, norm64(x, None, gamma)[2], "f32", 4e-6 * 6, "y")
    q, _ = blank(1, 11, cols, torch.float8_e4m3fn)
    scale = torch.zeros(1, 11, device="cuda")
    call("lipz_rms_norm", L.lipz_rms_norm_args(
        dtype=0, y_dtype=L.LIPZ_FP8, cells=1, rows=11, cols=cols, eps=EPS, x=mat(x), y=mat(q), gamma=gamma.data_ptr(),
        gamma_cell=cols, y_scale=scale.data_ptr()))
    nan = torch.isnan(q.float()).all(2)[0].cpu().tolist()
    assert nan == [i == 4 for i in range(11)] == torch.isnan(scale)[0].cpu().tolist()
    assert not torch.isnan(q.float())[0, 5].any()


def grads64(h, rstd, gamma, dy, dh):
    h, dy, rstd = h.double(), dy.double(), rstd.double()[:, :, None]
    u, xh = dy * gamma.double()[:, None], h * rstd
    dx = rstd * (u - xh * (u * xh).mean(2, keepdim=True)) + (dh.double() if dh is not None else 0)
    size = (rstd * (u.abs() + xh.abs() * (u * xh).abs().mean(2, keepdim=True))).amax(2, keepdim=True)
    return dx, (dy * xh).sum(1), (dy * xh).abs().sum(1), size  # size: what dx's terms measure before they cancel


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("cols", COLS)
def test_norm_backward(cols, dtype):
    dt, code = TYPES[dtype][:2]
    g = torch.Generator(device="cuda").manual_seed(cols + 1)
    for cells, rows, res, pad, off in ((1, 1, True, 0, 0), (3, 5, False, 3, 1), (2, 300 if cols < 5000 else 37, True, 8, 0)):
        print(f"[case] norm backward {dtype} cols={cols} cells={cells} rows={rows}", flush=True)
        h = padded(g, cells, rows, cols, dt, pad, 1.5, off)
        dy = padded(g, cells, rows, cols, dt, pad + 1, 0.3)
        dh = padded(g, cells, rows, cols, dt, pad, 0.3) if res else None
        gamma = 1 + 0.1 * torch.randn(cells, cols, generator=g, device="cuda")
        rstd = torch.rsqrt(h.float().square().mean(2) + EPS)
        dx, dx_ok = blank(cells, rows, cols, dt, 3)
        dg = torch.full((cells, cols + 2), 7.0, device="cuda")
        a = L.lipz_rms_norm_backward_args(
            dtype=code, cells=cells, rows=rows, cols=cols, h=mat(h), dy=mat(dy), dh=mat(dh), dx=mat(dx),
            gamma=gamma.data_ptr(), gamma_cell=cols, rstd=rstd.data_ptr(), dgamma=dg.data_ptr(), dgamma_cell=cols + 2)
        call("lipz_rms_norm_backward", a)
        edx, edg, adg, size = grads64(h, rstd, gamma, dy, dh)
        close(dx, edx, dtype, 4e-6 * size + 2.0 ** -24 * edx.abs() + 1e-9, "dx")
        close(dg[:, :cols], edg, "f32", 1e-6 * adg + 1e-9, "dgamma")
        assert dx_ok() and bool((dg[:, cols:] == 7.0).all())
        first = dg.clone()
        call("lipz_rms_norm_backward", a)
        assert torch.equal(dg, first)  # sums in a fixed order
        # dx over dy, without dgamma
        a.dx, a.dgamma = mat(dy), None
        call("lipz_rms_norm_backward", a)
        assert torch.equal(dy, dx)


def test_norm_gradient_is_the_slope_of_the_norm():
    """sum(y dy) along a direction: differences of the fp32 forward against the backward's product."""
    g = torch.Generator(device="cuda").manual_seed(9)
    cells, rows, cols = 2, 3, 97
    x, dy, d = (torch.randn(cells, rows, cols, generator=g, device="cuda") for _ in range(3))
    gamma = 1 + 0.1 * torch.randn(cells, cols, generator=g, device="cuda")
    dgm = torch.randn(cells, cols, generator=g, device="cuda")

    def forward(x, gamma):
        y, rstd = torch.empty_like(x), torch.empty(cells, rows, device="cuda")
        call("lipz_rms_norm", L.lipz_rms_norm_args(
            dtype=0, y_dtype=0, cells=cells, rows=rows, cols=cols, eps=EPS, x=mat(x), y=mat(y), gamma=gamma.data_ptr(),
            gamma_cell=cols, rstd=rstd.data_ptr()))
        return (y.double() * dy.double()).sum().item(), rstd

    _, rstd = forward(x, gamma)
    dx, dg = torch.empty_like(x), torch.empty(cells, cols, device="cuda")
    call("lipz_rms_norm_backward", L.lipz_rms_norm_backward_args(
        dtype=0, cells=cells, rows=rows, cols=cols, h=mat(x), dy=mat(dy), dx=mat(dx), gamma=gamma.data_ptr(),
        gamma_cell=cols, rstd=rstd.data_ptr(), dgamma=dg.data_ptr(), dgamma_cell=cols))
    t = 2.0 ** -7
    # the difference's own error: t^2 / 6 of the third derivative (about the slope's size here) and fp32 rounding / t
    got = (forward(x + t * d, gamma)[0] - forward(x - t * d, gamma)[0]) / (2 * t)
    want = (dx.double() * d.double()).sum().item()
    assert abs(got - want) < 2e-3 * max(1.0, dx.double().norm().item() * d.double().norm().item() / 10)
    got = (forward(x, gamma + t * dgm)[0] - forward(x, gamma - t * dgm)[0]) / (2 * t)
    assert abs(got - (dg.double() * dgm.double()).sum().item()) < 1e-3


def test_no_rows():
    y = torch.empty(0, device="cuda")
    one = torch.ones(8, device="cuda")
    dg = torch.full((2, 4), 7.0, device="cuda")
    m = L.lipz_mat(one.data_ptr(), 4, 0)
    call("lipz_rms_norm", L.lipz_rms_norm_args(dtype=0, y_dtype=0, cells=2, rows=0, cols=4, eps=EPS, x=m, y=m,
                                               gamma=one.data_ptr(), gamma_cell=4))
    call("lipz_rms_norm_backward", L.lipz_rms_norm_backward_args(
        dtype=0, cells=2, rows=0, cols=4, h=m, dy=m, dx=m, gamma=one.data_ptr(), gamma_cell=4, rstd=one.data_ptr(),
        dgamma=dg.data_ptr(), dgamma_cell=4))
    assert bool((dg == 0).all()) and bool((one == 1).all()) and y.numel() == 0
