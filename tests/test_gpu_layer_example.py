"""The operators of a layer together, as examples/dense_layer.py uses them: it runs, and its gradients are the formulas'."""
import importlib.util
import math
import os

import pytest
import torch

import layer_ref as ref
import paper_2505_11170_amd as gws
from gated_ref import assert_within
from gpu_util import DEV, ensure_built

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "dense_layer.py")


@pytest.fixture(scope="module")
def example():
    ensure_built()
    spec = importlib.util.spec_from_file_location("dense_layer", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_it_runs(example):
    said = []
    losses, layer, x = example.train(512, 256, 768, 6, say=said.append)
    assert len(losses) == 6 and all(math.isfinite(v) and v > 0 for v in losses) and len(said) == 7
    assert 0.0 < float(layer.clip[0]) and 0.0 < float(layer.clip[1]) <= 1.0
    for d in layer.desc.values():
        assert bool(torch.isfinite(d.w.float()).all())
    # a token alone is the row of the batch, but for the order of the sums: two roundings of N and H on either side, one of Y
    y = layer.forward(x)[:1].clone()
    one = layer.token(x[:1])
    wu, wd = (layer.desc[n].w_hat.double() for n in ("up", "down"))
    h, z = layer.h[:1].double(), layer.z[:1].double()
    dz = layer.n[:1].double().abs() @ wu.abs().t() * 2.0 ** -7 + z.abs() * 2.0 ** -20
    size = (1.2 * dz + h.abs() * 2.0 ** -7) @ wd.abs().t()
    assert_within(one, y.double(), size + 2.0 ** -7 * y.double().abs() + 1e-6, "token")
    with pytest.raises(ValueError, match="multiple of 64"):
        example.DenseLayer(100, 256, 256)


def test_gradients_of_a_step(example):
    """Every result of the backward pass from what it was given, in 64 bits: one rounding of it (2^-8 relative), and what its inputs' roundings bring."""
    M, C, F = 320, 256, 512
    layer = example.DenseLayer(M, C, F, seed=5)
    gen = torch.Generator(device=DEV).manual_seed(6)
    x, dy = torch.randn(M, C, generator=gen, device=DEV).bfloat16(), (torch.randn(M, C, generator=gen, device=DEV) * 1e-2).bfloat16()
    for v in layer.vectors.values():
        v += 0.1 * torch.randn(v.shape, generator=gen, device=DEV)
    layer.sample(3)
    layer.forward(x)
    dx = layer.backward(x, dy, 3).double()
    r, t24 = 2.0 ** -8, 2.0 ** -24
    wu, wd, g = layer.desc["up"].w_hat.double(), layer.desc["down"].w_hat.double(), layer.vectors["gamma"].double()
    a, slope = ref.act(gws.ACT_GELU_TANH, layer.z.double())
    d, n = dy.double(), layer.n.double()
    dh, dh_size = d @ wd, d.abs() @ wd.abs()
    long = 2 * max(M, F) * t24                                   # of a sum's additions in fp32
    dz = dh * slope
    tol = r * dz.abs() + (long + 2.0 ** -18) * 1.2 * dh_size
    assert_within(layer.dz, dz, tol, "dz")
    assert_within(layer.grads["b_up"], dz.sum(0), ((long + 2.0 ** -18) * 1.2 * dh_size).sum(0) + long * dz.abs().sum(0), "b_up")
    assert_within(layer.grads["b_down"], d.sum(0), long * d.abs().sum(0), "b_down")
    h, dzk = layer.h.double(), layer.dz.double()
    for name, left, right in (("down", d, h), ("up", dzk, n)):
        want, size = left.t() @ right, left.abs().t() @ right.abs()
        assert_within(layer.desc[name].dw, want, r * want.abs() + long * size, "dw " + name)
    # through the norm, from the statistics in 64 bits: dn is BF16 (in the layer's buffer), the statistics are fp32
    dn = layer.dn.double()
    want = dzk @ wu
    assert_within(layer.dn, want, r * want.abs() + long * (dzk.abs() @ wu.abs()), "dn")
    xd = x.double()
    mean = xd.mean(1, keepdim=True)
    rstd = 1.0 / ((xd - mean).square().mean(1, keepdim=True) + 1e-5).sqrt()
    hat, t = (xd - mean) * rstd, dn * g
    want = rstd * (t - t.mean(1, keepdim=True) - hat * (t * hat).mean(1, keepdim=True)) + d
    size = rstd * (t.abs() + t.abs().mean(1, keepdim=True) + hat.abs() * (t * hat).abs().mean(1, keepdim=True)) + d.abs()
    assert_within(dx, want, r * want.abs() + 4 * C * t24 * size, "dx")
    assert_within(layer.grads["gamma"], (dn * hat).sum(0), (2 * M + 2 * C) * t24 * (dn.abs() * (hat.abs() + 1.0)).sum(0), "gamma")
    assert_within(layer.grads["beta"], dn.sum(0), 2 * M * t24 * dn.abs().sum(0), "beta")


def test_the_gradient_against_differences(example):
    """Along one direction of each vector: the loss in 64 bits through the formulas, at weights as they were sampled."""
    M, C, F = 64, 256, 256
    layer = example.DenseLayer(M, C, F, seed=8)
    gen = torch.Generator(device=DEV).manual_seed(9)
    x, dy = torch.randn(M, C, generator=gen, device=DEV).bfloat16(), torch.randn(M, C, generator=gen, device=DEV).bfloat16()
    layer.sample(1)
    layer.forward(x)
    layer.backward(x, dy, 1)
    wu, wd = (layer.desc[k].w_hat.double() for k in ("up", "down"))

    def loss(v):
        xd = x.double()
        c = xd - xd.mean(1, keepdim=True)
        n = c / (c.square().mean(1, keepdim=True) + 1e-5).sqrt() * v["gamma"] + v["beta"]
        return float((dy.double() * (ref.act(gws.ACT_GELU_TANH, n @ wu.t() + v["b_up"])[0] @ wd.t() + v["b_down"] + xd)).sum())

    start = {k: v.double() for k, v in layer.vectors.items()}
    for k, grad in layer.grads.items():
        step = torch.randn(grad.shape, generator=gen, device=DEV).double()
        e = 1e-4
        numeric = (loss({**start, k: start[k] + e * step}) - loss({**start, k: start[k] - e * step})) / (2 * e)
        analytic = float((grad.double() * step).sum())
        # BF16 roundings of N, H's input Z, dZ and dn, 2^-8 each, on sums of many terms of both signs: against the sum of the terms' sizes, not their sum
        size = float((grad.double() * step).abs().sum())
        assert abs(numeric - analytic) <= 4 * 2.0 ** -8 * size, (k, numeric, analytic, size)
