"""The gated block's operators together, as examples/gated_ffn.py uses them."""
import importlib.util
import os

import pytest
import torch

import gated_ref as ref
import paper_2505_11170_amd as gws
from gpu_util import ensure_built

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "gated_ffn.py")


@pytest.fixture(scope="module")
def example():
    ensure_built()
    spec = importlib.util.spec_from_file_location("gated_ffn", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_training_lowers_the_loss(example):
    losses, ffn, x = example.train(1024, 256, 512, 25, say=lambda *_: None)
    assert losses[-1] < 0.5 * losses[0], losses
    # a token alone: the row of the batch, but for the order of the sums
    y = ffn.forward(x)[:1].double().clone()
    one = ffn.token(x[:1])
    torch.cuda.synchronize()
    g, u, d = (ffn.desc[n].w_hat for n in ("gate", "up", "down"))
    h = ref.gate(ref.SILU, x[:1].double() @ g.double().t())[0] * (x[:1].double() @ u.double().t())
    bound = (h.abs() @ d.double().abs().t()) * 2.0 ** -7 + 2.0 ** -8 * y.abs()    # two roundings of H, one of Y, on either side
    ref.assert_within(one, h @ d.double().t(), bound, "token")
    ref.assert_within(y, h @ d.double().t(), bound, "row of the batch")


def test_a_step_against_64_bits(example):
    # every result of a backward pass from what that pass was given: bounds as in the tests of each operator, put together
    M, K, F = 512, 256, 512
    ffn = example.GatedFFN(M, K, F, seed=5)
    ffn.sample(1)
    gen = torch.Generator(device="cuda:0").manual_seed(6)
    x = torch.randn(M, K, generator=gen, device="cuda:0").bfloat16()
    dy = (torch.randn(M, K, generator=gen, device="cuda:0") * 1e-3).bfloat16()
    ffn.forward(x)
    dx = ffn.backward(dy, 1)
    torch.cuda.synchronize()
    wg, wu, wd = (ffn.desc[n].w_hat.double() for n in ("gate", "up", "down"))
    g, u = ref.decode(ffn.saved.g8.codes, ffn.saved.g8.xscale), ref.decode(ffn.saved.u8.codes, ffn.saved.u8.xscale)
    xv = ref.decode(ffn.x8.codes, ffn.x8.xscale)
    a, slope = ref.gate(ref.SILU, g)
    dh = dy.double() @ wd
    dg, du, h = dh * u * slope, dh * a, a * u
    r = 2.0 ** -8
    near = lambda got, want, size, what: ref.assert_within(got, want, r * want.abs() + 2 * r * size, what)  # noqa: E731
    near(dx, dg @ wg + du @ wu, dg.abs() @ wg.abs() + du.abs() @ wu.abs(), "dx")
    near(ffn.desc["gate"].dw, dg.t() @ xv, dg.abs().t() @ xv.abs(), "dw gate")
    near(ffn.desc["up"].dw, du.t() @ xv, du.abs().t() @ xv.abs(), "dw up")
    near(ffn.desc["down"].dw, dy.double().t() @ h, dy.double().abs().t() @ h.abs(), "dw down")
    for n in ("gate", "up", "down"):
        dbt = ffn.desc[n].dbt.clone()
        gws.gws_sample_bwd([gws.TensorDesc(rows=ffn.desc[n].rows, cols=ffn.desc[n].cols, seed=ffn.desc[n].seed, g=ffn.desc[n].dw, scale=ffn.desc[n].scale,
                                           dbt=ffn.desc[n].dbt)], 1)
        torch.cuda.synchronize()
        scale = float(dbt.abs().max())
        assert scale > 0 and float((dbt - ffn.desc[n].dbt).abs().max()) <= 1e-5 * scale
