"""The example's residual networks: gradients against automatic differentiation in 64 bits, training, scoring in 8 bits.

Tolerances.  fp32: a gradient passes through at most 8 operators here, each within 4e-6 of the sum of its terms'
magnitudes; 1e-4 of the tensor's largest value leaves an order for terms that cancel.  e4m3: a rounding of a value in
3 explicit bits is off by 2^-4 of it at most, uniformly by 2^-4 / sqrt(3) / sqrt(2) = 2.6 % in the root mean square
(averaged over a binade); x and w each, so 3.6 % of a product's norm, over 4 layers that do not add up to more than
their sum: 15 %."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
spec = importlib.util.spec_from_file_location("residual_blocks", os.path.join(ROOT, "examples", "residual_blocks.py"))
rb = importlib.util.module_from_spec(spec)
spec.loader.exec_module(rb)


def reference(x, params, blocks):
    def norm(h, gamma):
        return h / torch.sqrt((h * h).mean(2, keepdim=True) + rb.EPS) * gamma[:, None]

    def layer(l, h):
        gamma, w, b = params[l]
        return torch.bmm(norm(h, gamma), w) + b[:, None]

    h = torch.nn.functional.silu(layer(0, x))
    for l in range(1, blocks + 1):
        h = h + torch.nn.functional.silu(layer(l, h))
    return layer(blocks + 1, h) + x


@pytest.mark.parametrize("blocks", [0, 1, 2, 3])
def test_gradients(blocks):
    nets = rb.ResidualNets(3, 37, 24, blocks, 11, "f32", seed=blocks)
    g = torch.Generator(device="cuda").manual_seed(5)
    for layer in nets.params:
        for p in (layer[0], layer[2]):
            p.add_(0.3 * torch.randn(p.shape, generator=g, device="cuda"))
    nets.x.copy_(torch.randn(nets.x.shape, generator=g, device="cuda"))
    nets.dy.copy_(torch.randn(nets.dy.shape, generator=g, device="cuda"))
    y, grads = nets.forward(), nets.backward()
    x = nets.x.double().cpu().requires_grad_(True)
    params = [tuple(p.double().cpu().requires_grad_(True) for p in layer) for layer in nets.params]
    want = reference(x, params, blocks)
    flat = [p for layer in params for p in layer]
    expect = torch.autograd.grad(want, [x] + flat, nets.dy.double().cpu())
    got = [nets.dx] + [t for layer in grads for t in layer]
    for a, b in zip([y] + got, [want.detach()] + list(expect)):
        assert (a.double().cpu() - b).abs().max() <= 1e-4 * b.abs().max()


def test_scoring_in_8_bits():
    nets = rb.ResidualNets(2, 100, 96, 2, 33, "bf16", seed=1)
    g = torch.Generator(device="cuda").manual_seed(6)
    nets.x.copy_(torch.randn(nets.x.shape, generator=g, device="cuda"))
    y = (nets.forward() - nets.x).double()  # without the input that both add
    nets.quantize()
    y8 = (nets.score() - nets.x).double()
    assert 0 < (y8 - y).norm() <= 0.15 * y.norm()


def test_training(capsys):
    first, mse, mse8 = rb.main(["--cells", "4", "--width", "64", "--blocks", "2", "--batch", "50", "--steps", "120"])
    assert mse < 0.8 * first and abs(mse8 - mse) < 0.25 * mse
