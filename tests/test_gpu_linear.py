"""lipz_linear, lipz_linear_backward, lipz_quantize_weights and lipz_linear_fp8 against the formulas in 64 bits, through
the C ABI.

Tolerances.  A sum of n products p in fp32: 2^-23 (16 + 2 sqrt(n)) sum |p|, well above the sqrt(n) 2^-24 of rounding
errors that do not conspire and far below a lost product's 1 / n share for the n here.  Activations: 1e-6 (1 + |z|) for
their own evaluation, slopes at most 1.2.  The backward pass rounds dz to the type: each rounding is off by at most
2^-8 (bf16) or 2^-11 (f16) of its dz, so a sum of them by 6 times the root of the summed squares (over ten standard
deviations).  On top, half a unit in the last place of the output's type."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_1811_12843_amd as L  # noqa: E402

from block_harness import TYPES, blank, call, close, mat, padded  # noqa: E402

SLOPE = 0.2
ACTS = ["linear", "relu", "lrelu", "tanh", "gelu", "silu"]
CODE = dict(L.ACTS, gelu=L.LIPZ_ACT_GELU, silu=L.LIPZ_ACT_SILU)
ROUND = {"f32": 0.0, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}

# cells, rows, fan_in, fan_out: single elements and rows, odd sizes, whole tiles, tiles' edges, sums split over a long
# axis, many cells on the larger tiles
SIZES = [(1, 1, 1, 1), (2, 1, 16, 8), (3, 3, 5, 7), (1, 1, 300, 1000), (2, 5, 2049, 72), (2, 17, 33, 65), (1, 64, 64, 64),
         (1, 65, 129, 63), (2, 130, 64, 257), (1, 16, 4096, 48), (1, 9, 8200, 136), (1, 1000, 40, 24), (16, 300, 100, 500),
         (48, 300, 96, 260), (1, 520, 1032, 776), (5, 2, 24, 4100)]


def act64(name, z):
    if name == "gelu":
        return z * torch.special.ndtr(z)
    if name == "silu":
        return z * torch.sigmoid(z)
    return {"linear": lambda: z, "relu": lambda: z.clamp_min(0), "tanh": lambda: torch.tanh(z),
            "lrelu": lambda: torch.where(z > 0, z, SLOPE * z)}[name]()


def slope64(name, z):
    if name == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "silu":
        return torch.sigmoid(z) * (1 + z * torch.sigmoid(-z))
    return {"linear": lambda: torch.ones_like(z), "relu": lambda: (z > 0).double(), "tanh": lambda: 1 - torch.tanh(z) ** 2,
            "lrelu": lambda: torch.where(z > 0, 1.0, SLOPE).double()}[name]()


def off(x, w):
    """The tolerance of the fp32 sums of x @ w."""
    n = x.shape[2]
    return 2.0 ** -23 * (16 + 2 * math.sqrt(n)) * torch.bmm(x.double().abs(), w.double().abs())


def forward(x, w, b, r, act, pre, y, cells=None):
    C, M, K = x.shape
    kind = {t[0]: t[1] for t in TYPES.values()}[x.dtype]
    call("lipz_linear", L.lipz_linear_args(
        dtype=kind, cells=C, rows=M, fan_in=K, fan_out=w.shape[2], act=CODE[act], slope=SLOPE, x=mat(x), w=mat(w),
        residual=mat(r), pre=mat(pre), y=mat(y), bias=b.data_ptr() if b is not None else None,
        bias_cell=b.stride(0) if b is not None else 0))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_linear(size, dtype):
    C, M, K, N = size
    dt = TYPES[dtype][0]
    g = torch.Generator(device="cuda").manual_seed(K + N)
    for k, (pad, at) in enumerate(((0, 0), (8, 0), (3, 1))):
        act, other = ACTS[(K + k) % 6], (K + N + k) % 3
        print(f"[case] linear {dtype} {size} pad={pad} offset={at} {act}", flush=True)
        x, w = padded(g, C, M, K, dt, pad, 1.0, at), padded(g, C, K, N, dt, pad, K ** -0.5)
        b = torch.randn(C, N + 3, generator=g, device="cuda")[:, :N] if other != 1 else None
        r = padded(g, C, M, N, dt, pad + 1) if other != 2 else None
        y, y_ok = blank(C, M, N, dt, 3)
        pre, pre_ok = blank(C, M, N, dt, 8 * k)
        forward(x, w, b, r, act, pre if other else None, y)
        z = torch.bmm(x.double(), w.double())
        t = off(x, w)
        if b is not None:
            z = z + b.double()[:, None]
            t = t + 2.0 ** -23 * z.abs()
        want = act64(act, z) + (r.double() if r is not None else 0)
        if other:
            close(pre, z, dtype, t, "pre")
        close(y, want, dtype, 1.2 * t + 1e-6 * (1 + z.abs()) + 2.0 ** -23 * want.abs(), "y")
        assert y_ok() and pre_ok()


def backward(x, w, pre, dy, act, dx, dw, db):
    C, M, N = dy.shape
    kind = {t[0]: t[1] for t in TYPES.values()}[dy.dtype]
    K = x.shape[2] if x is not None else w.shape[1]
    a = L.lipz_linear_backward_args(
        dtype=kind, cells=C, rows=M, fan_in=K, fan_out=N, act=CODE[act], slope=SLOPE, x=mat(x), w=mat(w), pre=mat(pre),
        dy=mat(dy), dx=mat(dx), dw=mat(dw), db=db.data_ptr() if db is not None else None,
        db_cell=db.stride(0) if db is not None else 0)
    call("lipz_linear_backward", a)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_linear_backward(size, dtype):
    C, M, K, N = size
    dt = TYPES[dtype][0]
    g = torch.Generator(device="cuda").manual_seed(K + N + 1)
    for k, (pad, at) in enumerate(((0, 0), (8, 0), (3, 1))):
        act = ACTS[(K + k) % 6]
        print(f"[case] linear backward {dtype} {size} pad={pad} offset={at} {act}", flush=True)
        x, w = padded(g, C, M, K, dt, pad, 1.0, at), padded(g, C, K, N, dt, pad, K ** -0.5, at)
        pre, dy = padded(g, C, M, N, dt, pad), padded(g, C, M, N, dt, pad, 1.0, at)
        dx, dx_ok = blank(C, M, K, dt, 5)
        dw, dw_ok = blank(C, K, N, dt, 5)
        db = torch.full((C, N + 2), 7.0, device="cuda")
        backward(x, w, pre if act != "linear" else None, dy, act, dx, dw, db)
        s = slope64(act, pre.double())
        dz = dy.double() * s
        near = 2e-6 * dy.double().abs() * (1 + pre.double().abs())  # dz before its rounding
        if act == "linear":
            near, rnd = torch.zeros_like(dz), 0.0
        else:
            rnd = ROUND[dtype]
        wt, xt = w.double().mT.contiguous(), x.double().mT.contiguous()

        def tol(a, b, da, db):
            sq = torch.bmm(a * a, b * b).sqrt()
            return off(a, b) + torch.bmm(da, db) + 6 * rnd * sq + 2.0 ** -24 * a.shape[2] ** 0.5  # (f16: subnormal dz)

        close(dx, torch.bmm(dz, wt), dtype, tol(dz, wt, near, wt.abs()), "dx")
        close(dw, torch.bmm(xt, dz), dtype, tol(xt, dz, xt.abs(), near), "dw")
        close(db[:, :N], dz.sum(1), "f32",
              2.0 ** -23 * (16 + 2 * math.sqrt(M)) * dz.abs().sum(1) + near.sum(1) + 1e-30, "db")
        assert dx_ok() and dw_ok() and bool((db[:, N:] == 7.0).all())
        # each gradient alone is the same, and so is a second call
        for which in range(3):
            d1, d2, d3 = (torch.full_like(t, 7.0) for t in (dx, dw, db))
            backward(x if which == 1 else None, w if which != 1 else None, pre if act != "linear" else None, dy, act,
                     d1 if which == 0 else None, d2 if which == 1 else None, d3 if which == 2 else None)
            assert torch.equal((d1, d2, d3[:, :N])[which], (dx, dw, db[:, :N])[which])


def test_linear_in_place_shared_and_beside():
    """y over the residual; x and w shared by the cells; the cells' outputs side by side in a row."""
    g = torch.Generator(device="cuda").manual_seed(5)
    C, M, K, N = 3, 50, 72, 40
    x, w = torch.randn(1, M, K, generator=g, device="cuda"), torch.randn(1, K, N, generator=g, device="cuda") / 8
    b, r = torch.randn(C, N, generator=g, device="cuda"), torch.randn(M, C, N, generator=g, device="cuda")
    want = act64("tanh", torch.bmm(x.double(), w.double()) + b.double()[:, None]) + r.transpose(0, 1).double()
    y = r.transpose(0, 1)
    forward(x.expand(C, M, K), w.expand(C, K, N), b, y, "tanh", None, y)
    close(y, want, "f32", 2 * off(x, w) + 4e-6, "y")


def test_linear_bad_values_stay_in_their_rows_and_columns():
    g = torch.Generator(device="cuda").manual_seed(6)
    for dt in (torch.float32, torch.bfloat16, torch.float16):
        for K, N in ((100, 100), (64, 72)):
            x, w = padded(g, 1, 70, K, dt, 2), padded(g, 1, K, N, dt, 2)
            x[0, 7, K - 1], w[0, 0, 9] = float("nan"), float("inf")
            y, _ = blank(1, 70, N, dt, 1)
            forward(x, w, None, None, "linear", None, y)
            bad = ~torch.isfinite(y[0].float())
            assert bool(bad[7].all()) and bool(bad[:, 9].all())
            bad[7], bad[:, 9] = False, False
            assert not bool(bad.any())


def test_linear_offsets_past_32_bits():
    """Rows 2^20 elements apart: the last ones lie over 4 GiB from the first."""
    M, K, N, ld = 2600, 64, 48, 1 << 20
    g = torch.Generator(device="cuda").manual_seed(7)
    big = torch.empty(M * ld, dtype=torch.bfloat16, device="cuda")
    x = big.as_strided((1, M, K), (M * ld, ld, 1))
    y = big.as_strided((1, M, N), (M * ld, ld, 1), 4096)
    x.copy_(torch.randn(1, M, K, generator=g, device="cuda"))
    w = (torch.randn(1, K, N, generator=g, device="cuda") / 8).bfloat16()
    forward(x, w, None, None, "relu", None, y)
    z = torch.bmm(x.double(), w.double())
    close(y, z.clamp_min(0), "bf16", off(x, w), "y")
    dx = big.as_strided((1, M, K), (M * ld, ld, 1), 8192)
    dw = torch.empty_like(w)
    backward(x, w, y, y, "relu", dx, dw, None)
    dz = y.double()  # relu' is 1 where y > 0, and y is 0 elsewhere
    close(dx, torch.bmm(dz, w.double().mT.contiguous()), "bf16", off(dz, w.double().mT.contiguous()), "dx")
    close(dw, torch.bmm(x.double().mT.contiguous(), dz), "bf16", off(x.double().mT.contiguous(), dz), "dw")


def test_linear_no_rows():
    one = torch.ones(64, device="cuda")
    m, none = L.lipz_mat(one.data_ptr(), 8, 0), L.lipz_mat()
    call("lipz_linear", L.lipz_linear_args(dtype=0, cells=2, rows=0, fan_in=8, fan_out=8, x=m, w=m, y=m, slope=SLOPE))
    call("lipz_linear_fp8", L.lipz_linear_fp8_args(y_dtype=0, cells=2, rows=0, fan_in=8, fan_out=8, x=m, w=m, y=m,
                                                   x_scale=one.data_ptr(), w_scale=one.data_ptr()))
    assert bool((one == 1).all())
    for dt, kind in ((torch.float32, 0), (torch.bfloat16, 1), (torch.float16, 2)):
        dw, ok = blank(2, 8, 5, dt, 3)
        db = torch.full((2, 7), 7.0, device="cuda")
        call("lipz_linear_backward", L.lipz_linear_backward_args(
            dtype=kind, cells=2, rows=0, fan_in=8, fan_out=5, act=CODE["silu"], slope=SLOPE, x=m, w=m, pre=m, dy=m, dx=m,
            dw=mat(dw), db=db.data_ptr(), db_cell=7))
        assert bool((dw == 0).all()) and bool((db[:, :5] == 0).all()) and bool((db[:, 5:] == 7).all()) and ok()
    assert none.p is None


def test_linear_gradient_is_the_slope_of_the_product():
    """sum(y dy) along a direction: differences of the fp32 forward against the backward's products."""
    g = torch.Generator(device="cuda").manual_seed(8)
    C, M, K, N = 2, 9, 21, 13
    x, ex = (torch.randn(C, M, K, generator=g, device="cuda") for _ in range(2))
    w, ew = (torch.randn(C, K, N, generator=g, device="cuda") / 4 for _ in range(2))
    b, eb = (torch.randn(C, N, generator=g, device="cuda") for _ in range(2))
    dy = torch.randn(C, M, N, generator=g, device="cuda")
    for act in ("linear", "tanh", "gelu", "silu"):
        def loss(t):
            y = torch.empty(C, M, N, device="cuda")
            forward(x + t * ex, w + t * ew, b + t * eb, None, act, None, y)
            return (y.double() * dy.double()).sum().item()

        pre, y = torch.empty(C, M, N, device="cuda"), torch.empty(C, M, N, device="cuda")
        forward(x, w, b, None, act, pre, y)
        dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
        backward(x, w, pre, dy, act, dx, dw, db)
        want = sum((p.double() * q.double()).sum().item() for p, q in ((dx, ex), (dw, ew), (db, eb)))
        t = 2.0 ** -8
        # the difference's own error: t^2 / 6 of the third derivative, and the sums' fp32 rounding (234 of 1e-6) / t
        assert abs((loss(t) - loss(-t)) / (2 * t) - want) < 0.02 + 1e-3 * abs(want)


# ---- e4m3 ----

@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("size", [(1, 1, 1), (3, 5, 7), (2, 64, 64), (1, 300, 130), (2, 257, 65), (1, 1032, 520)],
                         ids=lambda s: "x".join(map(str, s)))
def test_quantize_weights(size, dtype):
    C, K, N = size
    dt, kind = TYPES[dtype][:2]
    g = torch.Generator(device="cuda").manual_seed(K)
    for pad in (0, 3):
        print(f"[case] quantize {dtype} {size} pad={pad}", flush=True)
        w = padded(g, C, K, N, dt, pad, 0.1)
        w[0, :, 0] = 0
        q, ok = blank(C, N, K, torch.float8_e4m3fn, pad)
        scale = torch.full((C, N + 1), 7.0, device="cuda")
        a = L.lipz_quantize_weights_args(dtype=kind, cells=C, fan_in=K, fan_out=N, w=mat(w), q=mat(q),
                                         scale=scale.data_ptr(), scale_cell=N + 1)
        call("lipz_quantize_weights", a)
        want = torch.clamp_min(w.double().abs().amax(1) / 448, 2.0 ** -126)
        close(scale[:, :N], want, "f32", 2.0 ** -24 * want, "scale")  # 1 / 448 is rounded, then the product
        # the quotient by the fp32 scale, once rounded in fp32
        close(q, w.double().mT / scale[:, :N].double()[:, :, None], "fp8", 448 * 2.0 ** -24, "q")
        assert ok() and bool((scale[:, N] == 7).all())
        w[C - 1, K // 2, N - 1] = float("nan") if pad else float("inf")
        call("lipz_quantize_weights", a)
        bad = torch.isnan(q.float())
        assert bool(bad[C - 1, N - 1].all()) and int(bad.sum()) == K and int(torch.isnan(scale).sum()) == 1


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_linear_fp8(size, dtype):
    C, M, K, N = size
    dt, kind = TYPES[dtype][:2]
    g = torch.Generator(device="cuda").manual_seed(K + N + 2)
    for k, (pad, at) in enumerate(((0, 0), (16, 0), (3, 1))):
        act, other = ACTS[(K + k) % 6], (K + N + k) % 3
        print(f"[case] linear_fp8 {dtype} {size} pad={pad} offset={at} {act}", flush=True)
        x, w = padded(g, C, M, K, torch.float8_e4m3fn, pad, 50.0, at), padded(g, C, N, K, torch.float8_e4m3fn, pad, 50.0)
        xs = (torch.rand(C, M + 1, generator=g, device="cuda") * 0.02 + 0.01)[:, :M]
        ws = (torch.rand(C, N + 2, generator=g, device="cuda") * (0.02 * K ** -0.5))[:, :N]
        b = torch.randn(C, N, generator=g, device="cuda") if other != 1 else None
        r = padded(g, C, M, N, dt, pad + 1) if other != 2 else None
        y, y_ok = blank(C, M, N, dt, 3)
        call("lipz_linear_fp8", L.lipz_linear_fp8_args(
            y_dtype=kind, cells=C, rows=M, fan_in=K, fan_out=N, act=CODE[act], slope=SLOPE, x=mat(x), w=mat(w),
            residual=mat(r), y=mat(y), x_scale=xs.data_ptr(), x_scale_cell=M + 1, w_scale=ws.data_ptr(),
            w_scale_cell=N + 2, bias=b.data_ptr() if b is not None else None, bias_cell=N))
        wt = w.double().mT.contiguous()
        s = xs.double()[:, :, None] * ws.double()[:, None]
        z, t = torch.bmm(x.double(), wt) * s, off(x, wt) * s
        if b is not None:
            z = z + b.double()[:, None]
        want = act64(act, z) + (r.double() if r is not None else 0)
        close(y, want, dtype, 1.2 * t + 1e-6 * (1 + z.abs()) + 2.0 ** -23 * want.abs(), "y")
        assert y_ok()


def test_block_on_another_stream_and_in_a_graph():
    """Norm, quantised weights and product on a side stream; then captured, and replayed on new inputs."""
    g = torch.Generator(device="cuda").manual_seed(10)
    C, M, D = 2, 40, 256
    h = torch.randn(C, M, D, generator=g, device="cuda").bfloat16()
    w = (torch.randn(C, D, D, generator=g, device="cuda") / 16).bfloat16()
    gamma = torch.ones(C, D, device="cuda")
    q, ws = torch.empty(C, D, D, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(C, D, device="cuda")
    n, ns = torch.empty(C, M, D, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(C, M, device="cuda")
    y, z = torch.empty_like(h), torch.empty_like(h)
    calls = []

    def add(name, args):
        nb = getattr(L, name + "_workspace_bytes")(args)
        calls.append((getattr(L, name), args, torch.empty(nb, dtype=torch.uint8, device="cuda"), nb))

    add("lipz_quantize_weights", L.lipz_quantize_weights_args(dtype=1, cells=C, fan_in=D, fan_out=D, w=mat(w), q=mat(q),
                                                              scale=ws.data_ptr(), scale_cell=D))
    add("lipz_rms_norm", L.lipz_rms_norm_args(dtype=1, y_dtype=3, cells=C, rows=M, cols=D, eps=1e-5, x=mat(h), y=mat(n),
                                              gamma=gamma.data_ptr(), gamma_cell=D, y_scale=ns.data_ptr()))
    add("lipz_linear_fp8", L.lipz_linear_fp8_args(
        y_dtype=1, cells=C, rows=M, fan_in=D, fan_out=D, act=CODE["gelu"], slope=SLOPE, x=mat(n), w=mat(q), residual=mat(h),
        y=mat(y), x_scale=ns.data_ptr(), x_scale_cell=M, w_scale=ws.data_ptr(), w_scale_cell=D))
    add("lipz_linear", L.lipz_linear_args(dtype=1, cells=C, rows=M, fan_in=D, fan_out=D, act=CODE["silu"], slope=SLOPE,
                                          x=mat(y), w=mat(w), y=mat(z)))

    def all_calls():
        s = torch.cuda.current_stream().cuda_stream
        for fn, args, work, nb in calls:
            fn(args, work.data_ptr(), nb, s)

    all_calls()
    torch.cuda.synchronize()
    want = y.clone(), z.clone()
    assert bool(torch.isfinite(z.float()).all())
    side = torch.cuda.Stream()
    y.zero_(), z.zero_()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        all_calls()
    side.synchronize()
    assert torch.equal(y, want[0]) and torch.equal(z, want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        all_calls()
    for k in range(4):
        h.copy_(torch.randn(C, M, D, generator=g, device="cuda"))
        y.zero_(), z.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone(), z.clone()
        all_calls()
        torch.cuda.synchronize()
        assert torch.equal(y, got[0]) and torch.equal(z, got[1]), k


# The largest tiles (two hundred and more of 256 x 256) with sums of many slices, odd ends on every side.
WIDE = [(48, 300, 1032, 260), (48, 257, 2085, 511), (1, 3585, 1040, 3586)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("size", WIDE, ids=lambda s: "x".join(map(str, s)))
def test_linear_on_the_largest_tiles(size, dtype):
    C, M, K, N = size
    dt, kind = TYPES[dtype][:2]
    g = torch.Generator(device="cuda").manual_seed(K)
    print(f"[case] largest tiles {dtype} {size}", flush=True)
    x, w = padded(g, C, M, K, dt, 8), padded(g, C, K, N, dt, 6, K ** -0.5)
    b, r = torch.randn(C, N, generator=g, device="cuda"), padded(g, C, M, N, dt, 2)
    y, y_ok = blank(C, M, N, dt, 3)
    pre, pre_ok = blank(C, M, N, dt)
    forward(x, w, b, r, "gelu", pre, y)
    z = torch.bmm(x.double(), w.double()) + b.double()[:, None]
    t = off(x, w) + 2.0 ** -23 * z.abs()
    want = act64("gelu", z) + r.double()
    close(pre, z, dtype, t, "pre")
    close(y, want, dtype, 1.2 * t + 1e-6 * (1 + z.abs()) + 2.0 ** -23 * want.abs(), "y")
    assert y_ok() and pre_ok()
    dx, dx_ok = blank(C, M, K, dt, 5)
    dw, dw_ok = blank(C, K, N, dt, 5)
    db = torch.empty(C, N, device="cuda")
    backward(x, w, None, r, "linear", dx, dw, db)
    wt, xt, dz = w.double().mT.contiguous(), x.double().mT.contiguous(), r.double()
    close(dx, torch.bmm(dz, wt), dtype, off(dz, wt), "dx")
    close(dw, torch.bmm(xt, dz), dtype, off(xt, dz), "dw")
    close(db, dz.sum(1), "f32", 2.0 ** -23 * (16 + 2 * math.sqrt(M)) * dz.abs().sum(1), "db")
    assert dx_ok() and dw_ok()


@pytest.mark.parametrize("size", WIDE, ids=lambda s: "x".join(map(str, s)))
def test_linear_fp8_on_the_largest_tiles(size):
    C, M, K, N = size
    g = torch.Generator(device="cuda").manual_seed(K + 1)
    print(f"[case] largest tiles e4m3 {size}", flush=True)
    x, w = padded(g, C, M, K, torch.float8_e4m3fn, 7, 50.0), padded(g, C, N, K, torch.float8_e4m3fn, 9, 50.0)
    xs, ws = torch.rand(C, M, generator=g, device="cuda") * 0.02 + 0.01, torch.rand(C, N, generator=g, device="cuda") * 1e-3
    y, y_ok = blank(C, M, N, torch.bfloat16, 3)
    call("lipz_linear_fp8", L.lipz_linear_fp8_args(
        y_dtype=L.LIPZ_BF16, cells=C, rows=M, fan_in=K, fan_out=N, act=CODE["silu"], slope=SLOPE, x=mat(x), w=mat(w),
        y=mat(y), x_scale=xs.data_ptr(), x_scale_cell=M, w_scale=ws.data_ptr(), w_scale_cell=N))
    wt, s = w.double().mT.contiguous(), xs.double()[:, :, None] * ws.double()[:, None]
    z, t = torch.bmm(x.double(), wt) * s, off(x, wt) * s
    close(y, act64("silu", z), "bf16", 1.2 * t + 1e-6 * (1 + z.abs()), "y")
    assert y_ok()
