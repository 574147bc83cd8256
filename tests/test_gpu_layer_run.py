"""The norms, the dense layer, the AdamW step and what they stand beside, as a training step uses them: against autograd in 64 bits, in captured graphs, on
streams, two calls at once."""
import math

import pytest
import torch

import layer_ref as ref
import paper_2505_11170_amd as gws
from gpu_util import DEV, ensure_built
from test_gpu_adamw import Parameter
from test_gpu_dense import weight
from test_gpu_gated import rand, room
from test_gpu_norm import vec

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_built()


class Layer:
    """y = x + gelu(norm(x) W1 + b1) W2 + b2 with all its buffers; weights stored [in x out]."""

    def __init__(self, M, C, F, kind, seed=0):
        self.M, self.C, self.F, self.kind = M, C, F, kind
        self.x = rand(seed + 1, M, C)
        self.w1, self.w2 = rand(seed + 2, C, F, C ** -0.5), rand(seed + 3, F, C, F ** -0.5)
        self.b1, self.b2, self.gamma, self.beta = vec(seed + 4, F, 0.0, 0.1), vec(seed + 5, C, 0.0, 0.1), vec(seed + 6, C, 1.0, 0.1), vec(seed + 7, C, 0.0, 0.1)
        b = lambda n: torch.zeros(M, n, dtype=torch.bfloat16, device=DEV)  # noqa: E731
        f = lambda n: torch.zeros(n, device=DEV)  # noqa: E731
        self.n, self.z, self.h, self.y, self.dz, self.dn, self.dx = b(C), b(F), b(F), b(C), b(F), b(C), b(C)
        self.mean, self.rstd, self.db1, self.db2, self.dgamma, self.dbeta = f(M), f(M), f(F), f(C), f(C), f(C)
        self.dw1, self.dw2 = torch.zeros_like(self.w1), torch.zeros_like(self.w2)
        size = max(gws.gws_norm_bwd_workspace_bytes(M, C), gws.gws_dense_bwd_workspace_bytes(M, max(C, F)))
        self.ws = torch.empty(size, dtype=torch.uint8, device=DEV)
        self.layer = kind == gws.NORM_LAYER

    def forward(self):
        gws.gws_norm_fwd(self.x, self.n, self.kind, gamma=self.gamma, beta=self.beta if self.layer else None, mean=self.mean if self.layer else None, rstd=self.rstd)
        gws.gws_dense_fwd(self.n, self.w1, self.h, bias=self.b1, act=gws.ACT_GELU_TANH, z=self.z)
        gws.gws_dense_fwd(self.h, self.w2, self.y, bias=self.b2, residual=self.x)
        return self.y

    def backward(self, dy):
        gws.gws_dense_bwd_h(dy, None, None, dbias=self.db2, workspace=self.ws)
        gws.gws_dense_bwd(dy, self.w2, self.z, self.dz, gws.ACT_GELU_TANH, h=self.h, dbias=self.db1, workspace=self.ws)
        if self.M % 64 == 0:
            gws.gws_linear_bwd_w(self.h, dy, gws.TensorDesc(rows=self.F, cols=self.C, seed=0, dw=self.dw2), 0)
            gws.gws_linear_bwd_w(self.n, self.dz, gws.TensorDesc(rows=self.C, cols=self.F, seed=0, dw=self.dw1), 0)
        gws.gws_gemm_bf16(self.dz, self.w1, self.dn, w_is_nk=True)
        gws.gws_norm_bwd(self.dn, self.x, self.dx, self.rstd, self.kind, mean=self.mean if self.layer else None, gamma=self.gamma, residual=dy, dgamma=self.dgamma,
                         dbeta=self.dbeta if self.layer else None, workspace=self.ws)

    def outputs(self):
        return [self.n, self.z, self.h, self.y, self.dz, self.dn, self.dx, self.mean, self.rstd, self.db1, self.db2, self.dgamma, self.dbeta, self.dw1, self.dw2]


@pytest.mark.parametrize("M,C,F", [(64, 256, 512), (1000, 256, 1024), (2048, 768, 2048)])
@pytest.mark.parametrize("kind", [gws.NORM_LAYER, gws.NORM_RMS])
def test_a_layer_against_autograd(M, C, F, kind):
    """Gradients of the layer against autograd of its definition in 64 bits.  Between the calls values are rounded to BF16 (norm, h, z, dz, dn: 2^-9 of their sizes
    each, as rounding errors of either sign); five such steps, each carried on through sums of hundreds of them, whose parts add as their squares: a gradient is within
    5 x 2^-9 of the norm of all of it, and by elements within six times that of the root mean square."""
    l = Layer(M, C, F, kind)
    dy = rand(99, M, C)
    l.forward()
    l.backward(dy)
    p = {k: getattr(l, k).double().requires_grad_() for k in ("x", "w1", "w2", "b1", "b2", "gamma", "beta")}
    mean = p["x"].mean(1, keepdim=True) if l.layer else 0.0
    d = p["x"] - mean
    n = d / torch.sqrt((d * d).mean(1, keepdim=True) + 1e-5) * p["gamma"] + (p["beta"] if l.layer else 0.0)
    z = n @ p["w1"] + p["b1"]
    y = p["x"] + z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)) @ p["w2"] + p["b2"]
    y.backward(dy.double())
    pairs = [(l.y, y.detach()), (l.dx, p["x"].grad), (l.db1, p["b1"].grad), (l.db2, p["b2"].grad), (l.dgamma, p["gamma"].grad)]
    pairs += [(l.dbeta, p["beta"].grad)] if l.layer else []
    pairs += [(l.dw1, p["w1"].grad), (l.dw2, p["w2"].grad)] if M % 64 == 0 else []
    for got, want in pairs:
        err = got.double() - want
        assert err.norm() <= 5 * 2.0 ** -9 * want.norm(), (err.norm() / want.norm()).item()
        assert err.abs().max() <= 6 * 5 * 2.0 ** -9 * max(want.abs().max().item(), want.square().mean().sqrt().item())


def test_a_step_in_a_captured_graph():
    """Forward, backward, clipping and update captured and replayed, with eager calls of the same on other data between the replays."""
    l, other = Layer(192, 256, 512, gws.NORM_LAYER), Layer(192, 256, 512, gws.NORM_LAYER, seed=50)
    dy = rand(99, 192, 256)
    ps = [Parameter(1, 40, 96, True), Parameter(2, 33, 100), Parameter(3, 1, 777, g_fp32=True)]
    packed = gws.pack_adamw([p.desc for p in ps])
    out, ws = torch.zeros(2, device=DEV), torch.empty(gws.gws_grad_norm_workspace_bytes(packed), dtype=torch.uint8, device=DEV)
    start = [w.clone() for p in ps for w in p.wholes] + [s.xscale.clone() for p in ps if p.codes for s in (p.m, p.v)]
    wholes = [w for p in ps for w in p.wholes] + [s.xscale for p in ps if p.codes for s in (p.m, p.v)]

    def step():
        l.forward()
        l.backward(dy)
        gws.gws_grad_norm(packed, out, ws, max_norm=0.01)
        gws.gws_adamw(packed, lr=1e-3, step=5, grad_scale=out[1:])

    def restore():
        for w, s in zip(wholes, start):
            w.copy_(s)

    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in l.outputs() + wholes + [out]]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for replay in range(4):
        restore()
        for t in l.outputs():
            t.zero_()
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for k, (a, b) in enumerate(zip(l.outputs() + wholes + [out], want)):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), (replay, k)
        other.forward()                      # eager work of the same kind in between
        other.backward(dy)
        torch.cuda.synchronize()


def test_two_graphs_that_share_a_workspace_one_after_the_other():
    a, b = Layer(300, 256, 512, gws.NORM_LAYER), Layer(300, 256, 512, gws.NORM_RMS, seed=20)
    b.ws = a.ws
    dy = rand(99, 300, 256)
    want, graphs = [], []
    for l in (a, b):
        l.forward()
        l.backward(dy)
        torch.cuda.synchronize()
        want.append([t.clone() for t in l.outputs()])
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            l.forward()
            l.backward(dy)
        graphs.append(g)
    for _ in range(3):
        a.ws.fill_(255)                      # NaN
        for l, g in zip((a, b), graphs):
            for t in l.outputs():
                t.zero_()
            g.replay()
        torch.cuda.synchronize()
        for l, w in zip((a, b), want):
            assert all(torch.equal(x, y) for x, y in zip(l.outputs(), w))


def test_two_streams_at_once():
    ls = [Layer(500, 256, 1024, gws.NORM_LAYER, seed=30 * i) for i in range(2)]
    dy = rand(99, 500, 256)
    for l in ls:
        l.forward()
        l.backward(dy)
    torch.cuda.synchronize()
    want = [[t.clone() for t in l.outputs()] for l in ls]
    streams = [torch.cuda.Stream() for _ in ls]
    for _ in range(3):
        for l in ls:
            for t in l.outputs():
                t.zero_()
        torch.cuda.synchronize()
        for l, s in zip(ls, streams):
            with torch.cuda.stream(s):
                l.forward()
                l.backward(dy)
        torch.cuda.synchronize()
        for l, w in zip(ls, want):
            assert all(torch.equal(x, y) for x, y in zip(l.outputs(), w))
    # and by the argument, as an object and as a handle
    for given in (streams[0], int(streams[1].cuda_stream)):
        y = torch.zeros_like(ls[0].n)
        torch.cuda.synchronize()
        gws.gws_norm_fwd(ls[0].x, y, gamma=ls[0].gamma, beta=ls[0].beta, stream=given)
        torch.cuda.synchronize()
        assert torch.equal(y, ls[0].n)


def test_padded_batch():
    """Rows past the last token: zeros in, and nothing of them in the gradients of the parameters; rows past the call's stay as they are."""
    M, live, C = 128, 100, 256
    x, dy = rand(1, M, C), rand(2, M, C)
    y, mean, rstd = room(M, C)[0], torch.full((M,), 7.0, device=DEV), torch.full((M,), 7.0, device=DEV)
    gws.gws_norm_fwd(x[:live], y[:live], mean=mean[:live], rstd=rstd[:live])
    assert (y[live:] == 7).all() and (mean[live:] == 7).all() and (rstd[live:] == 7).all()
    x2, dy2 = x.clone(), dy.clone()
    x2[live:], dy2[live:] = 0, 0
    grads = []
    for m, xs, ds in ((live, x, dy), (M, x2, dy2)):
        mean, rstd = torch.zeros(m, device=DEV), torch.zeros(m, device=DEV)
        gws.gws_norm_fwd(xs[:m], y[:m], mean=mean, rstd=rstd)
        dx, dgamma, dbeta = room(m, C)[0], torch.zeros(C, device=DEV), torch.zeros(C, device=DEV)
        ws = torch.empty(gws.gws_norm_bwd_workspace_bytes(m, C), dtype=torch.uint8, device=DEV)
        gws.gws_norm_bwd(ds[:m], xs[:m], dx, rstd, mean=mean, dgamma=dgamma, dbeta=dbeta, workspace=ws)
        w, tol = ref.norm_bwd(dy[:live], x[:live], gws.NORM_LAYER, None, mean[:live], rstd[:live], None)
        assert ((dgamma - w[1]).abs() <= tol[1]).all() and ((dbeta - w[2]).abs() <= tol[2]).all()
        grads.append(dx[:live])
        assert (dx[live:] == 0).all()
    assert torch.equal(*grads)


def test_the_update_feeds_the_next_sampling():
    """The BF16 copy that the update writes is what the sampling reads, rows of a wider buffer among it."""
    rows, cols, ld = 64, 96, 104
    p = Parameter(1, rows, cols, True, ld=ld)
    gws.gws_adamw([p.desc], lr=1e-2, step=1)
    bt, scale = torch.full((2, 3), 6.0, device=DEV), torch.zeros(2, 3, device=DEV)
    hat, hat2 = torch.zeros(rows, ld, dtype=torch.bfloat16, device=DEV), torch.zeros(rows, cols, dtype=torch.bfloat16, device=DEV)
    gws.gws_sample_fwd([gws.TensorDesc(rows=rows, cols=cols, seed=3, w=p.w, w_hat=hat, bt=bt, scale=scale, ld=ld)], gws.FMT_FP8_E4M3, 1)
    gws.gws_sample_fwd([gws.TensorDesc(rows=rows, cols=cols, seed=3, w=p.p.bfloat16().contiguous(), w_hat=hat2, bt=bt, scale=scale)], gws.FMT_FP8_E4M3, 1)
    assert torch.equal(hat[:, :cols], hat2)


def test_serving_one_token():
    """One row through norm and dense layer gives what a batch gives for that row, within the order of the sums."""
    C, F = 2048, 512
    x, w, b = rand(1, 5, C), weight(2, C, F, True), vec(3, F)
    out = []
    for rows in (x, x[2:3]):
        n, y = room(rows.shape[0], C)[0], room(rows.shape[0], F)[0]
        gws.gws_norm_fwd(rows, n, gws.NORM_RMS)
        gws.gws_dense_fwd(n, w, y, bias=b, act=gws.ACT_SILU, w_is_nk=True)
        out.append((n, y))
    assert torch.equal(out[0][0][2:3], out[1][0])
    (z, y), (tz, ty) = ref.dense_fwd(out[1][0], w, True, b, gws.ACT_SILU, None)
    assert ((out[1][1] - y).abs() <= ty).all() and ((out[0][1][2:3] - y).abs() <= ty).all()


def test_tensors_of_another_device_are_refused():
    x = rand(1, 4, 64)
    with pytest.raises(ValueError, match="device"):
        gws.gws_norm_fwd(x, torch.zeros(4, 64, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="device"):
        gws.gws_norm_fwd(x, torch.zeros_like(x), gamma=torch.zeros(64))
