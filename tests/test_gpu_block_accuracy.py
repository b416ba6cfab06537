"""Accuracy of the residual-block operators where values of very different sizes meet, against the formulas in 64 bits.

Tolerances.  Sums: 2^-23 (16 + 2 sqrt(n)) sum |p| for n products p, as for sums in fp32 of any operands, and half a unit
in the last place of the output's type."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_1811_12843_amd as L  # noqa: E402

from block_harness import TYPES, blank, call, close, mat  # noqa: E402

F8 = torch.float8_e4m3fn


def outliers(kind, rows, K, g):
    """Rows of e4m3 values whose products with each other are led by a few: small ones of one sign, and 448 in places.
    one: a single place; groups: every 64th; signs: every 64th, one row's set in turn plus and minus."""
    v = 1 + torch.rand(2, rows, K, generator=g, device="cuda")
    if kind == "one":
        v[:, :, K // 3] = 448
    else:
        v[:, :, 5::64] = 448
    if kind == "signs":
        v[1, :, 5::128] = -448
    return v.to(F8)


@pytest.mark.parametrize("kind", ["one", "groups", "signs"])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
# on 64 x 64 tiles, with the sum split and whole; and on larger ones
@pytest.mark.parametrize("size", [(3, 1024, 70), (70, 8192, 136), (1030, 1040, 1100), (1800, 1101, 1700)],
                         ids=lambda s: "x".join(map(str, s)))
def test_e4m3_sums_with_outliers(size, dtype, kind):
    """The small products count as much as they do in an fp32 sum: x [M][K] of one row kind times w [N][K]."""
    M, K, N = size
    dt, code = TYPES[dtype][:2]
    g = torch.Generator(device="cuda").manual_seed(K + N)
    print(f"[case] e4m3 outliers {dtype} {size} {kind}", flush=True)
    both = outliers(kind, max(M, N), K, g)
    x, w = both[:1, :M].contiguous(), both[1:, :N].contiguous()
    # powers of two that keep every output in f16's range
    xs = torch.full((1, M), 2.0 ** -8, device="cuda")
    ws = torch.full((1, N), 2.0 ** -14, device="cuda")
    y, ok = blank(1, M, N, dt, 3)
    call("lipz_linear_fp8", L.lipz_linear_fp8_args(
        y_dtype=code, cells=1, rows=M, fan_in=K, fan_out=N, x=mat(x), w=mat(w), y=mat(y), x_scale=xs.data_ptr(),
        x_scale_cell=M, w_scale=ws.data_ptr(), w_scale_cell=N))
    wt = w.double().mT.contiguous()
    z, size1 = torch.bmm(x.double(), wt), torch.bmm(x.double().abs(), wt.abs())
    close(y, z * 2.0 ** -22, dtype, 2.0 ** -23 * (16 + 2 * math.sqrt(K)) * size1 * 2.0 ** -22, "y")
    assert ok()


CODE = dict(L.ACTS, gelu=L.LIPZ_ACT_GELU, silu=L.LIPZ_ACT_SILU)
SLOPE = 0.2


def act_and_slope(name, z):
    """act(z), act'(z) and the sums of the magnitudes of the terms that they are, on the CPU (z in 64 bits)."""
    if name == "gelu":
        cdf = 0.5 * torch.special.erfc(-z / math.sqrt(2))
        d = z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
        return z * cdf, cdf + d, (z * cdf).abs(), cdf + d.abs()
    if name == "silu":
        s, c = 1 / (1 + torch.exp(-z)), 1 / (1 + torch.exp(z))
        return z * s, s * (1 + z * c), (z * s).abs(), s * (1 + (z * c).abs())
    e = torch.exp(-2 * z.abs())
    d = 4 * e / (1 + e) ** 2
    return torch.tanh(z), d, torch.tanh(z).abs(), d


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("act", ["gelu", "silu", "tanh"])
def test_activations_and_slopes_keep_their_tails(act, dtype):
    """act(z) by a bias alone and act'(z) by a gradient of ones, z from -12 to 12.

    Tolerance, relative to the terms' sum: 2^-23 (16 + 2 z^2), a few roundings and functions of 1 or 2 units each, and
    for an exponential or erfc that of an argument near z^2 / 2 or 2 |z|; 16-bit types' own approximations 2e-6 more,
    far below their rounding."""
    dt, code = TYPES[dtype][:2]
    z = torch.arange(-12 * 64, 12 * 64 + 1, device="cuda") / 64.0
    N = z.numel()
    x, w = torch.zeros(1, 1, 1, device="cuda", dtype=dt), torch.ones(1, 1, N, device="cuda", dtype=dt)
    y, ok = blank(1, 1, N, dt, 3)
    call("lipz_linear", L.lipz_linear_args(
        dtype=code, cells=1, rows=1, fan_in=1, fan_out=N, act=CODE[act], slope=SLOPE, x=mat(x), w=mat(w), y=mat(y),
        bias=z.data_ptr(), bias_cell=N))
    own = 0.0 if dtype == "f32" else 2e-6

    def tol(z, terms):
        return (2.0 ** -23 * (16 + 2 * z * z) + own) * terms

    zd = z.double().cpu()
    a, _, terms, _ = act_and_slope(act, zd)
    close(y[0, 0], a, dtype, tol(zd, terms), "act")
    assert ok()
    pre, dy, db = z.to(dt).view(1, 1, N), torch.ones(1, 1, N, device="cuda", dtype=dt), torch.empty(1, N, device="cuda")
    call("lipz_linear_backward", L.lipz_linear_backward_args(
        dtype=code, cells=1, rows=1, fan_in=1, fan_out=N, act=CODE[act], slope=SLOPE, pre=mat(pre), dy=mat(dy),
        db=db.data_ptr(), db_cell=N))
    zd = pre[0, 0].double().cpu()
    _, d, _, terms = act_and_slope(act, zd)
    close(db[0], d, "f32", tol(zd, terms), "slope")


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("act", ["linear", "relu", "lrelu", "tanh", "gelu", "silu"])
def test_activations_and_slopes_at_infinity_are_their_limits(act, dtype):
    """Such as a pre-activation past the type's range, which is stored as an infinity.  NaN stays NaN."""
    dt, code = TYPES[dtype][:2]
    inf, nan = float("inf"), float("nan")
    far = 60000.0
    z = torch.tensor([inf, -inf, nan, far, -far], device="cuda")
    x, w = torch.zeros(1, 1, 1, device="cuda", dtype=dt), torch.ones(1, 1, 5, device="cuda", dtype=dt)
    y, pre = torch.empty(1, 1, 5, device="cuda", dtype=dt), torch.empty(1, 1, 5, device="cuda", dtype=dt)
    call("lipz_linear", L.lipz_linear_args(
        dtype=code, cells=1, rows=1, fan_in=1, fan_out=5, act=CODE[act], slope=0.25, x=mat(x), w=mat(w), pre=mat(pre),
        y=mat(y), bias=z.data_ptr(), bias_cell=5))
    db, dy = torch.empty(1, 5, device="cuda"), torch.ones(1, 1, 5, device="cuda", dtype=dt)
    call("lipz_linear_backward", L.lipz_linear_backward_args(
        dtype=code, cells=1, rows=1, fan_in=1, fan_out=5, act=CODE[act], slope=0.25, pre=mat(pre), dy=mat(dy),
        db=db.data_ptr(), db_cell=5))
    f = torch.tensor(far, device="cuda").to(dt).item()
    up = {"tanh": (1, 1)}.get(act, (inf, f))
    low = {"tanh": (-1, -1), "linear": (-inf, -f), "lrelu": (-inf, -f / 4)}.get(act, (0, 0))
    got = y[0, 0].float().tolist()
    assert math.isnan(got[2]) and got[:2] + got[3:] == [up[0], low[0], up[1], low[1]]
    above, below = (0 if act == "tanh" else 1), {"linear": 1, "lrelu": 0.25}.get(act, 0)
    got = db[0].tolist()
    assert got[:2] + got[3:] == [above, below] * 2 and (math.isnan(got[2]) or act == "linear")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [3, 40, 2000])  # (64 x 64 tiles with split and whole sums, 128 x 128 tiles)
def test_e4m3_scales_whose_product_leaves_the_range(rows, dtype):
    """z = x_scale w_scale sum, where x_scale w_scale alone is subnormal, 0 or infinite in fp32 and z is not; and sums of
    0 and scales of NaN."""
    dt, code = TYPES[dtype][:2]
    K, N = 1100, 1720
    g = torch.Generator(device="cuda").manual_seed(rows)
    for up in (False, True):
        size = 2.0 ** -5 if up else 100.0
        x, w = ((torch.randn(1, n, K, generator=g, device="cuda") * size).to(F8) for n in (rows, N))
        x[0, 1] = 0
        xs, ws = (1 + torch.rand(1, n, generator=g, device="cuda") for n in (rows, N))
        # sums near 2^18 (2^-5): z between 2^-120 and 2^-110 (2^105 and 2^125)
        xs, ws = xs * (2.0 ** 66 if up else 2.0 ** -70), ws * (2.0 ** 64 if up else 2.0 ** -62)
        xs[0, 0], ws[0, 0] = (xs[0, 0] * 2.0 ** -80, ws[0, 0] * 2.0 ** 40) if up else (2.0 ** -126, ws[0, 0])
        xs[0, 2], ws[0, 5] = float("nan"), float("nan")
        y, ok = blank(1, rows, N, dt, 3)
        print(f"[case] e4m3 scales {dtype} rows={rows} up={up}", flush=True)
        call("lipz_linear_fp8", L.lipz_linear_fp8_args(
            y_dtype=code, cells=1, rows=rows, fan_in=K, fan_out=N, x=mat(x), w=mat(w), y=mat(y), x_scale=xs.data_ptr(),
            x_scale_cell=rows, w_scale=ws.data_ptr(), w_scale_cell=N))
        wt, s = w.double().mT.contiguous(), xs.double()[:, :, None] * ws.double()[:, None]
        z, terms = torch.bmm(x.double(), wt) * s, torch.bmm(x.double().abs(), wt.abs()) * s
        far = torch.isinf(z.to(dt))  # past the type's range: an infinity
        z[far] = z[far] * float("inf")
        # (the sums' own tolerance, and a subnormal unit where z is that small)
        close(y, z, dtype, torch.nan_to_num(2.0 ** -23 * (16 + 2 * math.sqrt(K)) * terms) + 2.0 ** -149, "y")
        assert ok()
