"""Every kernel of the products of the residual-block operators on sums of many slices, against 64 bits: each type,
orientation and tile, with every count of slices left over by the pipeline's stages, odd ends on all sides.

Tolerances.  Sums of n products p: 2^-23 (16 + 2 sqrt(n)) sum |p|, and half a unit in the last place of the type."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_1811_12843_amd as L  # noqa: E402

from block_harness import TYPES, blank, call, close, mat, padded  # noqa: E402

# rows and columns that take a tile, and lengths of k: slices are 128 bytes of k (tiles of 256: 64), stages three on tiles of 64,
# four on the others
OUTPUTS = {64: (70, 75), 128: (1800, 1700), 256: (3970, 4000)}


def lengths(kind, tile):
    per = (64 if tile == 256 else 128) // {"f32": 4, "bf16": 2, "f16": 2, "fp8": 1}[kind]
    first = {64: 4, 128: {"f32": 20, "bf16": 12, "f16": 12, "fp8": 18}[kind], 256: 7}[tile]
    return [per * (first + i) - (0, per // 3, 1, per - 1)[i] for i in range(4)]


CASES = [(kind, tile, k) for kind in ("f32", "bf16", "f16") for tile in (64, 128, 256) if kind != "f32" or tile < 256
         for k in lengths(kind, tile)]


def tolerance(a, b):
    return 2.0 ** -23 * (16 + 2 * math.sqrt(a.shape[2])) * torch.bmm(a.abs(), b.abs())


def planned(kind, m, n, k, tile):
    assert L.lipz_test_product_plan(TYPES[kind][1], m, n, k)[0] == tile


@pytest.mark.parametrize("kind,tile,k", CASES, ids=lambda v: str(v))
def test_products(kind, tile, k):
    """x w, dy w^T and x^T dy, of k terms each."""
    M, N = OUTPUTS[tile]
    planned(kind, M, N, k, tile)
    dt, code = TYPES[kind][:2]
    g = torch.Generator(device="cuda").manual_seed(k)
    print(f"[case] products {kind} tiles of {tile} k={k}", flush=True)
    x, w = padded(g, 1, M, k, dt, 3), padded(g, 1, k, N, dt, 6, k ** -0.5)
    y, ok = blank(1, M, N, dt, 3)
    call("lipz_linear", L.lipz_linear_args(dtype=code, cells=1, rows=M, fan_in=k, fan_out=N, x=mat(x), w=mat(w), y=mat(y),
                                           slope=0.2))
    xd, wd = x.double(), w.double()
    close(y, torch.bmm(xd, wd), kind, tolerance(xd, wd), "y")
    assert ok()
    # dx [M][N] = dy [M][k] (w [N][k])^T
    dy, w = x, padded(g, 1, N, k, dt, 5, k ** -0.5)
    dx, ok = blank(1, M, N, dt, 1)
    call("lipz_linear_backward", L.lipz_linear_backward_args(
        dtype=code, cells=1, rows=M, fan_in=N, fan_out=k, act=0, slope=0.2, w=mat(w), dy=mat(dy), dx=mat(dx)))
    wt = w.double().mT.contiguous()
    close(dx, torch.bmm(xd, wt), kind, tolerance(xd, wt), "dx")
    assert ok()
    # dw [M][N] = x [k][M]^T dy [k][N]
    x, dy = padded(g, 1, k, M, dt, 2, k ** -0.5), padded(g, 1, k, N, dt, 4)
    dw, ok = blank(1, M, N, dt, 1)
    call("lipz_linear_backward", L.lipz_linear_backward_args(
        dtype=code, cells=1, rows=k, fan_in=M, fan_out=N, act=0, slope=0.2, x=mat(x), dy=mat(dy), dw=mat(dw)))
    xt, dyd = x.double().mT.contiguous(), dy.double()
    close(dw, torch.bmm(xt, dyd), kind, tolerance(xt, dyd), "dw")
    assert ok()


@pytest.mark.parametrize("out", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("tile,k", [(t, k) for t in (64, 128) for k in lengths("fp8", t)])
def test_products_of_e4m3(tile, k, out):
    M, N = OUTPUTS[tile]
    planned("fp8", M, N, k, tile)
    dt, code = TYPES[out][:2]
    g = torch.Generator(device="cuda").manual_seed(k)
    print(f"[case] products e4m3 {out} tiles of {tile} k={k}", flush=True)
    x, w = padded(g, 1, M, k, torch.float8_e4m3fn, 3, 50.0), padded(g, 1, N, k, torch.float8_e4m3fn, 9, 50.0)
    xs, ws = torch.rand(1, M, generator=g, device="cuda") * 0.02 + 0.01, torch.rand(1, N, generator=g, device="cuda") * 1e-3
    y, ok = blank(1, M, N, dt, 3)
    call("lipz_linear_fp8", L.lipz_linear_fp8_args(
        y_dtype=code, cells=1, rows=M, fan_in=k, fan_out=N, x=mat(x), w=mat(w), y=mat(y), x_scale=xs.data_ptr(),
        x_scale_cell=M, w_scale=ws.data_ptr(), w_scale_cell=N, slope=0.2))
    wt, s = w.double().mT.contiguous(), xs.double()[:, :, None] * ws.double()[:, None]
    z = torch.bmm(x.double(), wt) * s
    close(y, z, out, tolerance(x.double(), wt) * s + 2.0 ** -22 * z.abs(), "y")
    assert ok()


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16", "fp8"])
@pytest.mark.parametrize("size", [(9, 130, 5000), (130, 200, 90), (1800, 1700, 2600), (2300, 2300, 200), (3990, 4000, 200)],
                         ids=lambda s: "x".join(map(str, s)))
def test_over_the_residual(size, kind):
    """y in the residual's place: with the sum split, on each tile, an odd width's last columns among them."""
    M, N, K = size
    N += 3
    dt, code = TYPES["bf16" if kind == "fp8" else kind][:2]
    tile, splits = L.lipz_test_product_plan(TYPES[kind][1], M, N, K)
    g = torch.Generator(device="cuda").manual_seed(M)
    print(f"[case] over the residual {kind} {size} tiles of {tile}, {splits} splits", flush=True)
    r = padded(g, 1, M, N, dt, 1)
    apart, _ = blank(1, M, N, dt, 2)
    if kind == "fp8":
        x, w = padded(g, 1, M, K, TYPES[kind][0], 0, 50.0), padded(g, 1, N, K, TYPES[kind][0], 0, 50.0)
        xs, ws = torch.rand(1, M, generator=g, device="cuda") * 0.02, torch.rand(1, N, generator=g, device="cuda") * 1e-3

        def run(y):
            call("lipz_linear_fp8", L.lipz_linear_fp8_args(
                y_dtype=code, cells=1, rows=M, fan_in=K, fan_out=N, act=L.LIPZ_ACT_SILU, x=mat(x), w=mat(w), residual=mat(r),
                y=mat(y), x_scale=xs.data_ptr(), x_scale_cell=M, w_scale=ws.data_ptr(), w_scale_cell=N, slope=0.2))
    else:
        x, w = padded(g, 1, M, K, dt, 0), padded(g, 1, K, N, dt, 0, K ** -0.5)

        def run(y):
            call("lipz_linear", L.lipz_linear_args(
                dtype=code, cells=1, rows=M, fan_in=K, fan_out=N, act=L.LIPZ_ACT_SILU, slope=0.2, x=mat(x), w=mat(w),
                residual=mat(r), y=mat(y)))
    run(apart)
    run(r)
    assert torch.equal(r, apart)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("cols", [5, 37, 256, 1000, 2049, 5000, 16390])
def test_norm_gradient_over_the_skips(cols, kind):
    """dx in dh's place."""
    dt, code = TYPES[kind][:2]
    g = torch.Generator(device="cuda").manual_seed(cols)
    h, dy, dh = (padded(g, 2, 19, cols, dt, 1) for _ in range(3))
    gamma, rstd = torch.rand(2, cols, generator=g, device="cuda"), torch.rand(2, 19, generator=g, device="cuda")
    apart, _ = blank(2, 19, cols, dt, 2)
    for dx in (apart, dh):
        call("lipz_rms_norm_backward", L.lipz_rms_norm_backward_args(
            dtype=code, cells=2, rows=19, cols=cols, h=mat(h), dy=mat(dy), dh=mat(dh), dx=mat(dx), gamma=gamma.data_ptr(),
            gamma_cell=cols, rstd=rstd.data_ptr()))
    assert torch.equal(dh, apart)
