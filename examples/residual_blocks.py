"""Pre-norm residual networks, one per grid cell, trained and then scored in 8 bits: the residual-block operators together.

Each cell owns a network that takes a fainter second image off a flattened image, x -> x + W_out n_L + b_out, with

    h_0 = silu(norm(x) W_in + b_in),  a_l = silu(norm(h_l) W_l + b_l),  h_{l+1} = h_l + a_l,  n_L = norm(h_L)

Every product reads a norm's output.  The skip connections' additions are the norms' (lipz_rms_norm adds a_l to h_l while it
reads them), their gradients join in lipz_rms_norm_backward, and the output layer adds x in its epilogue.  Training keeps
fp32 master weights and updates them with Adam; the products read rounded copies.  Scoring quantises the weights once
(lipz_quantize_weights); the norms then write e4m3 rows with scales, and lipz_linear_fp8 multiplies them.

    python examples/residual_blocks.py [--cells 16] [--width 256] [--blocks 4] [--batch 100] [--steps 300] [--dtype bf16]
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_1811_12843_amd as L  # noqa: E402
import synth.datasets  # noqa: E402

EPS = 1e-5
TYPES = {"f32": (torch.float32, L.LIPZ_F32), "bf16": (torch.bfloat16, L.LIPZ_BF16), "f16": (torch.float16, L.LIPZ_F16)}


def mat(t):
    """The lipz_mat of a tensor [cells][rows][columns]; None: a matrix left out."""
    return L.lipz_mat() if t is None else L.lipz_mat(t.data_ptr(), t.stride(1), t.stride(0))


class Calls:
    """Operator calls in order, with one workspace: what runs on one stream may share it."""

    def __init__(self):
        self.calls, self.bytes, self.workspace = [], 0, None

    def add(self, name, args):
        need = getattr(L, name + "_workspace_bytes")(args)
        if not need:
            raise ValueError(f"{name}: invalid arguments")
        self.calls.append((getattr(L, name), args))
        self.bytes = max(self.bytes, need)

    def run(self):
        if self.workspace is None:
            self.workspace = torch.empty(self.bytes, dtype=torch.uint8, device="cuda")
        stream = torch.cuda.current_stream().cuda_stream
        for fn, args in self.calls:
            fn(args, self.workspace.data_ptr(), self.bytes, stream)


class ResidualNets:
    """The cells' networks for a fixed batch: parameters, buffers and the calls of each pass.

    `params` are the fp32 master weights, as (gamma [C][D], w [C][D][N], b [C][N]) per layer; `x` [C][batch][dim] is the
    input, `y` the output, `dy` the output's gradient (written by the caller before backward()), and `grads` the gradients
    in the parameters' order; `dx` is the input's."""

    def __init__(self, cells, dim, width, blocks, batch, dtype="bf16", seed=0):
        self.dt, self.code = TYPES[dtype]
        self.C, self.M = cells, batch
        g = torch.Generator(device="cuda").manual_seed(seed)
        sizes = [(dim, width)] + [(width, width)] * blocks + [(width, dim)]
        # branches start small, so that the network starts near the identity
        scales = [1.0] + [0.5] * blocks + [0.1]
        self.params = [(torch.ones(cells, k, device="cuda"),
                        torch.randn(cells, k, n, generator=g, device="cuda") * (s * k ** -0.5),
                        torch.zeros(cells, n, device="cuda")) for (k, n), s in zip(sizes, scales)]
        self.moments = [tuple((torch.zeros_like(p), torch.zeros_like(p)) for p in layer) for layer in self.params]
        self.steps = 0
        self.sizes = sizes
        self.w = [p[1].to(self.dt) for p in self.params]
        self.x, self.y, self.dy = self._buf(dim), self._buf(dim), self._buf(dim)
        # per layer: the norm's input sum h, its 1 / rms, its output n, the pre-activation, the layer's output a
        self.rstd = [torch.empty(cells, batch, device="cuda") for _ in sizes]
        self.n = [self._buf(k) for k, _ in sizes]
        self.pre = [self._buf(n) for _, n in sizes]
        self.a = [self._buf(n) for _, n in sizes[:-1]] + [self.y]
        self.h = [self.x, self.a[0]] + [self._buf(width) for _ in range(blocks)]
        self.grads = [(torch.empty_like(p[0]), torch.empty_like(w), torch.empty_like(p[2]))
                      for p, w in zip(self.params, self.w)]
        self._forward, self._backward = self._plan_forward(), self._plan_backward()
        self._quantize = self._score = None

    def _buf(self, cols, dtype=None):
        return torch.empty(self.C, self.M, cols, dtype=dtype or self.dt, device="cuda")

    def _act(self, l):
        return L.LIPZ_ACT_LINEAR if l == len(self.sizes) - 1 else L.LIPZ_ACT_SILU

    def _norm_args(self, l, y, y_code, y_scale=None):
        # from layer 2 on the norm adds the branch to the skip
        src, branch, h = (self.h[l], None, None) if l < 2 else (self.h[l - 1], self.a[l - 1], self.h[l])
        return L.lipz_rms_norm_args(
            dtype=self.code, y_dtype=y_code, cells=self.C, rows=self.M, cols=self.sizes[l][0], eps=EPS, x=mat(src),
            residual=mat(branch), h=mat(h), y=mat(y), gamma=self.params[l][0].data_ptr(), gamma_cell=self.sizes[l][0],
            rstd=self.rstd[l].data_ptr(), y_scale=y_scale.data_ptr() if y_scale is not None else None)

    def _plan_forward(self):
        c, last = Calls(), len(self.sizes) - 1
        for l, (k, n) in enumerate(self.sizes):
            c.add("lipz_rms_norm", self._norm_args(l, self.n[l], self.code))
            c.add("lipz_linear", L.lipz_linear_args(
                dtype=self.code, cells=self.C, rows=self.M, fan_in=k, fan_out=n, act=self._act(l), x=mat(self.n[l]),
                w=mat(self.w[l]), residual=mat(self.x if l == last else None),
                pre=mat(None if l == last else self.pre[l]), y=mat(self.a[l]), bias=self.params[l][2].data_ptr(),
                bias_cell=n))
        return c

    def _plan_backward(self):
        c, last, self._between = Calls(), len(self.sizes) - 1, []
        da, skip = self.dy, None  # gradients of the layer's output, and of h past the branch
        for l in range(last, -1, -1):
            k, n = self.sizes[l]
            gamma, w, b = self.grads[l]
            dn = self._buf(k)
            c.add("lipz_linear_backward", L.lipz_linear_backward_args(
                dtype=self.code, cells=self.C, rows=self.M, fan_in=k, fan_out=n, act=self._act(l), x=mat(self.n[l]),
                w=mat(self.w[l]), pre=mat(None if l == last else self.pre[l]), dy=mat(da), dx=mat(dn), dw=mat(w),
                db=b.data_ptr(), db_cell=n))
            dh = self._buf(k)
            c.add("lipz_rms_norm_backward", L.lipz_rms_norm_backward_args(
                dtype=self.code, cells=self.C, rows=self.M, cols=k, h=mat(self.h[l]), dy=mat(dn),
                dh=mat(skip), dx=mat(dh), gamma=self.params[l][0].data_ptr(), gamma_cell=k, rstd=self.rstd[l].data_ptr(),
                dgamma=gamma.data_ptr(), dgamma_cell=k))
            # h_l = h_{l-1} + a_{l-1} has one gradient for both; h_1 is a_0; x is also added to the output
            da, skip = dh, (dh if l >= 2 else self.dy)
            self._between += [dn, dh]
        self.dx = dh
        return c

    def forward(self):
        self._forward.run()
        return self.y

    def backward(self):
        self._backward.run()
        return self.grads

    def adam(self, lr=2e-3, beta1=0.9, beta2=0.999, eps=1e-8):
        self.steps += 1
        c1, c2 = 1 - beta1 ** self.steps, 1 - beta2 ** self.steps
        for params, grads, moments in zip(self.params, self.grads, self.moments):
            for p, g, (m, v) in zip(params, grads, moments):
                g = g.float()
                m.lerp_(g, 1 - beta1)
                v.lerp_(g * g, 1 - beta2)
                p.sub_(lr / c1 * m / ((v / c2).sqrt() + eps))
        for w, p in zip(self.w, self.params):
            w.copy_(p[1])

    # ---- scoring in 8 bits ----

    def quantize(self):
        """e4m3 copies of the present weights."""
        if self._quantize is None:
            f8 = torch.float8_e4m3fn
            self.q = [torch.empty(self.C, n, k, dtype=f8, device="cuda") for k, n in self.sizes]
            self.qs = [torch.empty(self.C, n, device="cuda") for _, n in self.sizes]
            self.n8 = [self._buf(k, f8) for k, _ in self.sizes]
            self.ns = torch.empty(self.C, self.M, device="cuda")
            self._quantize, self._score = Calls(), Calls()
            last = len(self.sizes) - 1
            for l, (k, n) in enumerate(self.sizes):
                self._quantize.add("lipz_quantize_weights", L.lipz_quantize_weights_args(
                    dtype=self.code, cells=self.C, fan_in=k, fan_out=n, w=mat(self.w[l]), q=mat(self.q[l]),
                    scale=self.qs[l].data_ptr(), scale_cell=n))
                self._score.add("lipz_rms_norm", self._norm_args(l, self.n8[l], L.LIPZ_FP8, self.ns))
                self._score.add("lipz_linear_fp8", L.lipz_linear_fp8_args(
                    y_dtype=self.code, cells=self.C, rows=self.M, fan_in=k, fan_out=n, act=self._act(l),
                    x=mat(self.n8[l]), x_scale=self.ns.data_ptr(), x_scale_cell=self.M, w=mat(self.q[l]),
                    w_scale=self.qs[l].data_ptr(), w_scale_cell=n, residual=mat(self.x if l == last else None),
                    y=mat(self.a[l]), bias=self.params[l][2].data_ptr(), bias_cell=n))
        self._quantize.run()

    def score(self):
        """forward() on the weights of the last quantize()."""
        self._score.run()
        return self.y


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--cells", type=int, default=16)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--blocks", type=int, default=4)
    ap.add_argument("--batch", type=int, default=100)
    ap.add_argument("--steps", type=int, default=300)
    ap.add_argument("--fainter", type=float, default=0.5, help="the second image's share")
    ap.add_argument("--dtype", choices=sorted(TYPES), default="bf16")
    a = ap.parse_args(argv)
    data = torch.from_numpy(synth.datasets.mnist_like(8192, seed=1)).cuda()
    nets = ResidualNets(a.cells, data.shape[1], a.width, a.blocks, a.batch, a.dtype)
    g = torch.Generator(device="cuda").manual_seed(2)

    def batch():
        clean, second = (data[torch.randint(len(data), (a.cells, a.batch), generator=g, device="cuda")] for _ in range(2))
        nets.x.copy_(clean + a.fainter * second)
        return clean

    seen = []
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    for _ in range(a.steps):
        clean = batch()
        off = nets.forward().float() - clean
        seen.append(off.square().mean())
        # the squared error's gradient per cell, 2 / (batch dim), here without the constant: Adam divides it out
        nets.dy.copy_(off)
        nets.backward()
        nets.adam()
    torch.cuda.synchronize()
    ms = (time.perf_counter() - t0) / a.steps * 1e3
    first, last = float(seen[0]), float(torch.stack(seen[-10:]).mean())
    clean = batch()
    mse = float((nets.forward().float() - clean).square().mean())
    nets.quantize()
    mse8 = float((nets.score().float() - clean).square().mean())
    print(f"{a.cells} cells, {a.blocks} blocks of {a.width}, batch {a.batch}, {a.dtype}: {ms:.2f} ms a step, mean squared "
          f"error {first:.4f} -> {last:.4f}; a fresh batch {mse:.4f}, in 8 bits {mse8:.4f}", flush=True)
    return first, mse, mse8


if __name__ == "__main__":
    main()
