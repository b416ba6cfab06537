"""Timed cases of the residual-block operators, through the C ABI's Python binding.

A pre-norm residual block of a cell's network is h' = h + act(norm(h) W + b):
a root-mean-square norm that also adds the skip connection, a matrix product
with bias, activation and residual in its epilogue, their gradients, and for
scoring many samples the same block with 8-bit operands.  Every operator takes
a leading axis of cells (each with its own parameters), as the grid's networks
have it.

  norm        h = x + residual, rstd, y = h rstd gamma (or y in e4m3 with a scale per row)
  norm_bwd    gradients of x and gamma
  linear      y = act(x w + b) + residual (and the pre-activation, where the backward pass wants it)
  linear_bwd  gradients of x, w and b
  fp8         y = act(sx sw (qx qw) + b) + residual on e4m3 operands; with "requant" the weights are
              quantised in the pass, as after a training step

  listed()            the cases; draw(rng) gives another of the same ranges
  prepare(case, seed) inputs, output buffers and (for the framework) the argument structs
  run(state)          one pass and its outputs
  work(case)          bytes and operations that a pass cannot do without
  exact(case, seed)   run's outputs in 64 bits
"""
import math

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_SIZE = {"f32": 4, "bf16": 2, "f16": 2, "fp8": 1}
_FP8 = torch.float8_e4m3fn
_FP8_MAX, _TINY, _EPS, _SLOPE = 448.0, 2.0 ** -126, 1e-5, 0.2


def listed():
    return [
        # one sample scored in 8 bits: the norm's smallest call, pure latency
        dict(name="norm_serve_row", do="norm", dtype="bf16", y="fp8", cells=1, rows=1, cols=4096, res=True, pad=0),
        # odd widths in 8 bits for a 3x3 grid's cells: rows off every vector width
        dict(name="norm_serve_cells", do="norm", dtype="f16", y="fp8", cells=9, rows=333, cols=2049, res=False, pad=2),
        # a wide block's norm in training, the largest call: bound by memory
        dict(name="norm_train_large", do="norm", dtype="bf16", y="bf16", cells=1, rows=16384, cols=4096, res=True, pad=0),
        # the norm's gradient for the 4x4 grid's hidden layers (16 cells, batch 100, width 256)
        dict(name="norm_bwd_cells", do="norm_bwd", dtype="f32", cells=16, rows=100, cols=256, res=True, pad=0),
        # and for a wide block
        dict(name="norm_bwd_large", do="norm_bwd", dtype="bf16", cells=1, rows=8192, cols=8192, res=True, pad=0),
        # one sample through a wide layer: the weights are read once, latency and memory
        dict(name="linear_serve_row", do="linear", dtype="bf16", cells=1, rows=1, k=4096, n=4096, act="silu", res=True,
             pre=False, pad=0),
        # the 4x4 grid's generator output layer (256 -> 784, batch 100) in fp32
        dict(name="linear_cells", do="linear", dtype="f32", cells=16, rows=100, k=256, n=784, act="tanh", res=False,
             pre=True, pad=0),
        # a wide layer in training: the largest product
        dict(name="linear_large", do="linear", dtype="bf16", cells=1, rows=8192, k=4096, n=8192, act="gelu", res=True,
             pre=True, pad=0),
        # gradients at odd sizes: no row is aligned
        dict(name="linear_bwd_ragged", do="linear_bwd", dtype="f16", cells=1, rows=1999, k=1201, n=777, act="lrelu", pad=0),
        # gradients of a wide layer
        dict(name="linear_bwd_large", do="linear_bwd", dtype="bf16", cells=1, rows=8192, k=4096, n=4096, act="silu", pad=0),
        # a handful of samples scored in 8 bits, the weights kept
        dict(name="fp8_serve", do="fp8", dtype="bf16", cells=1, rows=8, k=4096, n=8192, act="relu", res=True,
             requant=False, pad=0),
        # a large evaluation in 8 bits of weights that were just trained
        dict(name="fp8_large", do="fp8", dtype="bf16", cells=1, rows=8192, k=8192, n=4096, act="gelu", res=True,
             requant=True, pad=0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    do = rng.choice(["norm", "norm_bwd", "linear", "linear", "linear_bwd", "fp8"])
    even = rng.random() < 0.5  # widths that are multiples of 8, as most programs have them

    def width(lo, hi):
        v = _log_int(rng, lo, hi)
        return -(-v // 8) * 8 if even else v

    cells = 1 if rng.random() < 0.5 else _log_int(rng, 2, 64)
    c = dict(do=do, dtype=rng.choice(["f32", "bf16", "bf16", "f16"]), cells=cells, pad=rng.choice([0, 0, 0, 8, 5]))
    if do in ("norm", "norm_bwd"):
        c["cols"] = width(16, 16384)
        c["rows"] = _log_int(rng, 1, max(1, min(32768, (1 << 25) // (cells * c["cols"]))))
        c["res"] = rng.random() < 0.7
        if do == "norm":
            c["y"] = rng.choice([c["dtype"], "fp8"])
        return c
    c["k"], c["n"] = width(16, 8192), width(16, 8192)
    c["cells"] = cells = min(cells, max(1, (1 << 25) // (c["k"] * c["n"])))
    most = 2 ** 36 if c["dtype"] == "f32" else 2 ** 37
    most = min(16384, most // (2 * cells * c["k"] * c["n"]), (1 << 25) // (cells * (c["k"] + c["n"])))
    c["rows"] = _log_int(rng, 1, max(1, most))
    c["act"] = rng.choice(["linear", "relu", "lrelu", "tanh", "gelu", "silu"])
    if do != "linear_bwd":
        c["res"] = rng.random() < 0.5
    if do == "linear":
        c["pre"] = rng.random() < 0.5
    if do == "fp8":
        c["requant"] = rng.random() < 0.5
    return c


# ---- inputs ----

def _random(c, seed):
    """The inputs, as tensors [cells, rows, columns] of their types; rows are `pad` elements apart more than they are wide."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, C, M, pad = _DT[c["dtype"]], c["cells"], c["rows"], c["pad"]

    def normal(*shape, scale=1.0, dtype=dt):
        return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)

    def mat(rows, cols, scale=1.0):
        return normal(C, rows, cols + pad, scale=scale)[:, :, :cols]

    s = {}
    if c["do"] in ("norm", "norm_bwd"):
        D = c["cols"]
        s["gamma"] = 1 + normal(C, D, scale=0.1, dtype=torch.float32)
        if c["do"] == "norm":
            s["x"] = mat(M, D, 1.5)
            s["r"] = mat(M, D, 0.7) if c["res"] else None
        else:
            s["h"] = mat(M, D, 1.5)
            s["rstd"] = torch.rsqrt(s["h"].float().square().mean(2) + _EPS)
            s["dy"] = mat(M, D, 0.02)
            s["dh"] = mat(M, D, 0.02) if c["res"] else None
        return s
    K, N = c["k"], c["n"]
    s["b"] = normal(C, N, scale=0.1, dtype=torch.float32)
    if c["do"] == "fp8":
        s["x"], s["sx"] = _to_fp8(normal(C, M, K, dtype=torch.float32))
        w = mat(K, N, K ** -0.5)
        if c["requant"]:
            s["w"] = w
        else:
            s["q"], s["sw"] = _to_fp8(w.float().transpose(1, 2).contiguous())
        s["r"] = mat(M, N) if c["res"] else None
        return s
    s["x"] = mat(M, K)
    s["w"] = mat(K, N, K ** -0.5)
    if c["do"] == "linear":
        s["r"] = mat(M, N) if c["res"] else None
    else:
        s["pre"] = (torch.bmm(s["x"].float(), s["w"].float()) + s["b"][:, None]).to(dt)
        s["dy"] = mat(M, N, 0.02)
    return s


def _like(c, rows, cols, dtype):
    return torch.empty(c["cells"], rows, cols, dtype=dtype, device="cuda")


def prepare(case, seed):
    c = case
    s = dict(_random(c, seed), case=c)
    if own:
        s["plan"] = _plan(c, s)
    return s


def _plan(c, s):
    """Output buffers, workspace and argument structs: what a program of the framework keeps for a layer."""
    import paper_1811_12843_amd as L

    dt, C, M = _DT[c["dtype"]], c["cells"], c["rows"]
    code = {"f32": L.LIPZ_F32, "bf16": L.LIPZ_BF16, "f16": L.LIPZ_F16, "fp8": L.LIPZ_FP8}
    act = dict(L.ACTS, gelu=L.LIPZ_ACT_GELU, silu=L.LIPZ_ACT_SILU)

    def mat(t):
        return L.lipz_mat() if t is None else L.lipz_mat(t.data_ptr(), t.stride(1), t.stride(0))

    out, calls = {}, []

    def call(fn, args):
        nb = getattr(L, fn + "_workspace_bytes")(args)
        ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
        calls.append((getattr(L, fn), args, ws.data_ptr(), nb, ws))

    if c["do"] == "norm":
        D = c["cols"]
        out["rstd"] = torch.empty(C, M, device="cuda")
        out["y"] = _like(c, M, D, _FP8 if c["y"] == "fp8" else dt)
        if c["y"] == "fp8":
            out["scale"] = torch.empty(C, M, device="cuda")
        if c["res"]:
            out["h"] = _like(c, M, D, dt)
        call("lipz_rms_norm", L.lipz_rms_norm_args(
            dtype=code[c["dtype"]], y_dtype=code[c["y"]], cells=C, rows=M, cols=D, eps=_EPS, x=mat(s["x"]),
            residual=mat(s["r"]), h=mat(out.get("h")), y=mat(out["y"]), gamma=s["gamma"].data_ptr(), gamma_cell=D,
            rstd=out["rstd"].data_ptr(), y_scale=out["scale"].data_ptr() if "scale" in out else None))
    elif c["do"] == "norm_bwd":
        D = c["cols"]
        out["dx"], out["dgamma"] = _like(c, M, D, dt), torch.empty(C, D, device="cuda")
        call("lipz_rms_norm_backward", L.lipz_rms_norm_backward_args(
            dtype=code[c["dtype"]], cells=C, rows=M, cols=D, h=mat(s["h"]), dy=mat(s["dy"]), dh=mat(s["dh"]),
            dx=mat(out["dx"]), gamma=s["gamma"].data_ptr(), gamma_cell=D, rstd=s["rstd"].data_ptr(),
            dgamma=out["dgamma"].data_ptr(), dgamma_cell=D))
    elif c["do"] == "linear":
        K, N = c["k"], c["n"]
        out["y"] = _like(c, M, N, dt)
        if c["pre"]:
            out["pre"] = _like(c, M, N, dt)
        call("lipz_linear", L.lipz_linear_args(
            dtype=code[c["dtype"]], cells=C, rows=M, fan_in=K, fan_out=N, act=act[c["act"]], slope=_SLOPE,
            x=mat(s["x"]), w=mat(s["w"]), residual=mat(s["r"]), pre=mat(out.get("pre")), y=mat(out["y"]),
            bias=s["b"].data_ptr(), bias_cell=N))
    elif c["do"] == "linear_bwd":
        K, N = c["k"], c["n"]
        out["dx"], out["dw"], out["db"] = _like(c, M, K, dt), _like(c, K, N, dt), torch.empty(C, N, device="cuda")
        call("lipz_linear_backward", L.lipz_linear_backward_args(
            dtype=code[c["dtype"]], cells=C, rows=M, fan_in=K, fan_out=N, act=act[c["act"]], slope=_SLOPE,
            x=mat(s["x"]), w=mat(s["w"]), pre=mat(s["pre"]), dy=mat(s["dy"]), dx=mat(out["dx"]), dw=mat(out["dw"]),
            db=out["db"].data_ptr(), db_cell=N))
    else:
        K, N = c["k"], c["n"]
        q, sw = s.get("q"), s.get("sw")
        if c["requant"]:
            out["q"], out["sw"] = q, sw = _like(c, N, K, _FP8), torch.empty(C, N, device="cuda")
            call("lipz_quantize_weights", L.lipz_quantize_weights_args(
                dtype=code[c["dtype"]], cells=C, fan_in=K, fan_out=N, w=mat(s["w"]), q=mat(q), scale=sw.data_ptr(),
                scale_cell=N))
        out["y"] = _like(c, M, N, dt)
        call("lipz_linear_fp8", L.lipz_linear_fp8_args(
            y_dtype=code[c["dtype"]], cells=C, rows=M, fan_in=K, fan_out=N, act=act[c["act"]], slope=_SLOPE,
            x=mat(s["x"]), x_scale=s["sx"].data_ptr(), x_scale_cell=M, w=mat(q), w_scale=sw.data_ptr(), w_scale_cell=N,
            residual=mat(s["r"]), y=mat(out["y"]), bias=s["b"].data_ptr(), bias_cell=N))
    return out, calls


def run(state):
    if own:
        out, calls = state["plan"]
        stream = torch.cuda.current_stream().cuda_stream
        for fn, args, ws, nb, _ in calls:
            fn(args, ws, nb, stream)
        return out
    return _PLAIN[state["case"]["do"]](state["case"], state)


# ---- the plain forms: 32 bits, rounded once at the end ----

def _act(name, z):
    if name == "relu":
        return z.clamp_min(0)
    if name == "lrelu":
        return torch.where(z > 0, z, _SLOPE * z)
    if name == "tanh":
        return torch.tanh(z)
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _act_grad(name, z):
    """d act / d z."""
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "lrelu":
        return torch.where(z > 0, 1.0, _SLOPE).to(z.dtype)
    if name == "tanh":
        return 1 - torch.tanh(z).square()
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    if name == "silu":
        p = 1 / (1 + torch.exp(-z))
        return p * (1 + z * (1 - p))
    return torch.ones_like(z)


def _to_fp8(v):
    """e4m3 values and scales of fp32 rows."""
    scale = (v.abs().amax(2) / _FP8_MAX).clamp_min(_TINY)
    return (v / scale[:, :, None]).to(_FP8), scale


def _plain_norm(c, s):
    dt = _DT[c["dtype"]]
    h = s["x"].float()
    if c["res"]:
        h = h + s["r"].float()
    rstd = torch.rsqrt(h.square().mean(2) + _EPS)
    y = h * rstd[:, :, None] * s["gamma"][:, None]
    out = {"rstd": rstd}
    if c["y"] == "fp8":
        out["y"], out["scale"] = _to_fp8(y)
    else:
        out["y"] = y.to(dt)
    if c["res"]:
        out["h"] = h.to(dt)
    return out


def _plain_norm_bwd(c, s):
    rstd = s["rstd"][:, :, None]
    xh, dy = s["h"].float() * rstd, s["dy"].float()
    g = dy * s["gamma"][:, None]
    dx = rstd * (g - xh * (g * xh).mean(2, keepdim=True))
    if c["res"]:
        dx = dx + s["dh"].float()
    return {"dx": dx.to(_DT[c["dtype"]]), "dgamma": (dy * xh).sum(1)}


def _plain_linear(c, s):
    dt = _DT[c["dtype"]]
    z = torch.bmm(s["x"].float(), s["w"].float()) + s["b"][:, None]
    y = _act(c["act"], z)
    if c["res"]:
        y = y + s["r"].float()
    out = {"y": y.to(dt)}
    if c["pre"]:
        out["pre"] = z.to(dt)
    return out


def _plain_linear_bwd(c, s):
    dt = _DT[c["dtype"]]
    dz = s["dy"].float() * _act_grad(c["act"], s["pre"].float())
    return {"dx": torch.bmm(dz, s["w"].float().transpose(1, 2)).to(dt),
            "dw": torch.bmm(s["x"].float().transpose(1, 2), dz).to(dt), "db": dz.sum(1)}


def _plain_fp8(c, s):
    out, q, sw = {}, s.get("q"), s.get("sw")
    if c["requant"]:
        out["q"], out["sw"] = q, sw = _to_fp8(s["w"].float().transpose(1, 2).contiguous())
    z = torch.bmm(s["x"].float() * s["sx"][:, :, None], (q.float() * sw[:, :, None]).transpose(1, 2)) + s["b"][:, None]
    y = _act(c["act"], z)
    if c["res"]:
        y = y + s["r"].float()
    out["y"] = y.to(_DT[c["dtype"]])
    return out


_PLAIN = {"norm": _plain_norm, "norm_bwd": _plain_norm_bwd, "linear": _plain_linear, "linear_bwd": _plain_linear_bwd,
          "fp8": _plain_fp8}


# ---- what a pass cannot do without ----

def work(case):
    c = case
    C, M, e = c["cells"], c["rows"], _SIZE[c["dtype"]]
    if c["do"] == "norm":
        D, r = c["cols"], c["res"]
        return {"bytes": C * (M * D * (e * (1 + 2 * r) + _SIZE[c["y"]]) + 4 * D + 4 * M * (1 + (c["y"] == "fp8"))),
                "flops": C * M * D * (8 if c["y"] == "fp8" else 5)}
    if c["do"] == "norm_bwd":
        D = c["cols"]
        return {"bytes": C * (M * D * e * (3 + c["res"]) + 8 * D + 4 * M), "flops": C * M * D * 10}
    K, N = c["k"], c["n"]
    if c["do"] == "linear":
        return {"bytes": C * (e * (M * K + K * N + M * N * (1 + c["res"] + c["pre"])) + 4 * N), "flops": C * M * N * (2 * K + 4)}
    if c["do"] == "linear_bwd":
        pre = c["act"] != "linear"
        return {"bytes": C * (e * (2 * M * K + 2 * K * N + M * N * (1 + pre)) + 4 * N), "flops": C * M * N * (4 * K + 4)}
    quant = C * (K * N * (e + 1) + 4 * N) if c["requant"] else C * (K * N + 4 * N)
    return {"bytes": quant + C * (M * K + 4 * M + 4 * N + e * M * N * (1 + c["res"])), "flops": C * M * N * (2 * K + 6)}


# ---- the definitions in 64 bits ----

def _dbl(t):
    return None if t is None else t.double()


def _exact_act(name, z):
    if name == "gelu":  # z Phi(z)
        return z * torch.special.ndtr(z)
    if name == "silu":
        return z * torch.sigmoid(z)
    return {"linear": lambda v: v, "relu": torch.relu, "tanh": torch.tanh,
            "lrelu": lambda v: torch.where(v > 0, v, _SLOPE * v)}[name](z)


def _exact_slope(name, z):
    """d act / d z by automatic differentiation."""
    with torch.enable_grad():
        v = z.detach().clone().requires_grad_(True)
        return torch.autograd.grad(_exact_act(name, v).sum(), v)[0] if name != "linear" else torch.ones_like(z)


def _exact_scale(v):
    return torch.maximum(v.abs().max(2)[0] / _FP8_MAX, torch.full((), _TINY, dtype=torch.float64, device=v.device))


def exact(case, seed):
    c = case
    with torch.no_grad():
        s = _random(c, seed)
        if c["do"] == "norm":
            h = s["x"].double()
            if c["res"]:
                h = h + s["r"].double()
            rms = torch.sqrt((h * h).sum(2) / c["cols"] + _EPS)
            y = h / rms[:, :, None] * s["gamma"].double()[:, None]
            out = {"rstd": 1 / rms, "y": y}
            if c["y"] == "fp8":
                out["scale"] = _exact_scale(y)
                out["y"] = y / out["scale"][:, :, None]
            if c["res"]:
                out["h"] = h
            return out
        if c["do"] == "norm_bwd":
            h, dy, rstd = s["h"].double(), s["dy"].double(), s["rstd"].double()[:, :, None]
            u = dy * s["gamma"].double()[:, None]
            along = (u * h).sum(2, keepdim=True) / c["cols"]
            dx = rstd * u - rstd ** 3 * h * along
            if c["res"]:
                dx = dx + s["dh"].double()
            return {"dx": dx, "dgamma": (dy * h * rstd).sum(1)}
        if c["do"] == "linear":
            z = torch.baddbmm(s["b"].double()[:, None], s["x"].double(), s["w"].double())
            y = _exact_act(c["act"], z)
            if c["res"]:
                y = y + s["r"].double()
            return {"y": y, "pre": z} if c["pre"] else {"y": y}
        if c["do"] == "linear_bwd":
            dz = _exact_slope(c["act"], s["pre"].double()) * s["dy"].double()
            return {"dx": dz @ s["w"].double().mT, "dw": s["x"].double().mT @ dz, "db": dz.sum(1)}
        out, q, sw = {}, _dbl(s.get("q")), _dbl(s.get("sw"))
        if c["requant"]:
            w = s["w"].double().mT
            out["sw"] = _exact_scale(w)
            out["q"] = w / out["sw"][:, :, None]
            q, sw = _to_fp8(s["w"].float().mT.contiguous())  # the product is of the rounded weights
            q, sw = q.double(), sw.double()
        z = (s["x"].double() @ q.mT) * s["sx"].double()[:, :, None] * sw[:, None] + s["b"].double()[:, None]
        y = _exact_act(c["act"], z)
        if c["res"]:
            y = y + s["r"].double()
        out["y"] = y
        return out
