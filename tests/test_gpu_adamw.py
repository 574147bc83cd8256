"""The AdamW step and the gradients' norm: states to the bit (every fp32 operation is written out in layer_ref.py), parameters against 64 bits."""
import math

import numpy as np
import pytest
import torch

import layer_ref as ref
import paper_2505_11170_amd as gws
from gpu_util import DEV, ensure_built

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_built()


def padded(v, ld, dtype, fill=7):
    """`v` in rows of ld, what lies between them recognisable."""
    whole = torch.full((v.shape[0], ld), fill, dtype=dtype, device=DEV)
    whole[:, :v.shape[1]] = torch.as_tensor(v).to(DEV, dtype)
    return whole[:, :v.shape[1]], whole


def numbers(t):
    return t.float().cpu().numpy()


class Parameter:
    def __init__(self, seed, rows, cols, codes=False, g_fp32=False, ld=None, copy=True, decay=0.1, lr_scale=1.0, g=None, m=None, v=None):
        rng = np.random.default_rng(seed)
        ld = ld or -(-cols // 8) * 8
        self.rows, self.cols, self.codes, self.decay, self.lr_scale, self.seed = rows, cols, codes, decay, lr_scale, 0x1234567890ABCDEF * (seed + 1) % 2 ** 64
        shape = (rows, cols)
        n = lambda std: (rng.standard_normal(shape) * std * np.exp(rng.standard_normal((1, cols)))).astype(np.float32)  # noqa: E731
        self.wholes = []

        def put(x, dtype):
            t, whole = padded(x, ld, dtype)
            self.wholes.append(whole)
            return t

        self.p = put(n(0.02), torch.float32)
        self.g = put(n(1e-3) if g is None else g, torch.float32 if g_fp32 else torch.bfloat16)
        m, v = n(3e-4) if m is None else m, np.abs(n(1e-3)) if v is None else v
        if codes:
            half = np.full(shape, 0x8000)
            held = []
            for x, root in ((m, False), (v, True)):
                c, s = ref.encode_state(x, half, root)
                c, s = put(c, torch.uint8), torch.as_tensor(s).to(DEV)
                held.append(gws.Act8(c, s))
            self.m, self.v = held
        else:
            self.m, self.v = put(m, torch.float32), put(v * v, torch.float32)
        self.w = put(np.zeros(shape), torch.bfloat16) if copy else None
        self.desc = gws.AdamWTensor(p=self.p, g=self.g, m=self.m, v=self.v, w=self.w, weight_decay=decay, lr_scale=lr_scale, seed=self.seed)

    def state(self):
        if self.codes:
            return [ref.decode_state(a.codes.cpu().numpy(), a.xscale.cpu().numpy()).astype(np.float32) for a in (self.m, self.v)]
        return [numbers(self.m), numbers(self.v)]

    def before(self):
        self.old = (numbers(self.p), numbers(self.g), *self.state())

    def check(self, lr, step, beta1, beta2, eps, scale=1.0):
        p, g, m, v = self.old
        m1, v1, p1, tol = ref.adamw(p, g, m, v, self.codes, lr * np.float32(self.lr_scale), step, beta1, beta2, eps, np.float32(self.decay), scale)
        got = numbers(self.p).astype(np.float64)
        fine = np.isfinite(p1)
        assert (np.isfinite(got) == fine).all()
        assert (np.abs(got - p1)[fine] <= tol[fine]).all(), np.abs(got - p1)[fine].max()
        if self.w is not None:
            assert torch.equal(self.w.view(torch.int16)[torch.isfinite(self.p)], self.p.bfloat16().view(torch.int16)[torch.isfinite(self.p)])
        if self.codes:
            bits = ref.state_bits(self.rows, self.cols, self.seed, step)
            for a, x, b, root in ((self.m, m1, bits[0], False), (self.v, v1, bits[1], True)):
                codes, scales = ref.encode_state(x, b, root)
                assert (a.xscale.cpu().numpy() == scales).all(), "scales"
                assert (a.codes.cpu().numpy() == codes).all(), ("codes", root, np.argwhere(a.codes.cpu().numpy() != codes)[:4])
        else:
            assert np.array_equal(numbers(self.m), m1, equal_nan=True) and np.array_equal(numbers(self.v), v1, equal_nan=True)
        for whole in self.wholes:
            assert (whole[:, self.cols:].float() == 7).all()


SIZES = [(1, 1), (1, 3), (1, 31), (1, 768), (3, 33), (5, 100), (64, 96), (31, 257), (130, 1000), (257, 2048)]


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("g_fp32", [False, True])
def test_step(codes, g_fp32):
    ps = [Parameter(i, r, c, codes, g_fp32, ld=-(-c // 8) * 8 + (8 if i % 2 else 0), copy=i % 3 != 1, decay=0.1 * (i % 2), lr_scale=1.0 + i) for i, (r, c) in enumerate(SIZES)]
    for step in (1, 2, 1000, (1 << 33) + 5):
        for p in ps:
            p.before()
        gws.gws_adamw([p.desc for p in ps], lr=1e-3, step=step, beta1=0.9, beta2=0.999, eps=1e-8)
        for p in ps:
            p.check(1e-3, step, 0.9, 0.999, 1e-8)


def test_many_tensors_of_both_kinds_in_several_launches():
    ps = [Parameter(i, 1 + i % 7, 5 + 37 * (i % 11), codes=i % 3 == 0, g_fp32=i % 2 == 0) for i in range(130)]
    packed = gws.pack_adamw([p.desc for p in ps])
    scale = torch.tensor([0.37], device=DEV)
    for p in ps:
        p.before()
    gws.gws_adamw(packed, lr=3e-4, step=7, grad_scale=scale)
    for p in ps:
        p.check(3e-4, 7, 0.9, 0.95, 1e-8, scale=float(scale))


def test_many_vectors():
    """More than a launch holds, of fp32 states and next to each other; matrices without gaps among them."""
    ps = [Parameter(i, 1 if i % 5 else 3, 8 * (1 + i % 13) if i % 5 == 0 else 1 + 97 * (i % 17), g_fp32=i % 2 == 0, copy=i % 4 != 0) for i in range(260)]
    packed = gws.pack_adamw([p.desc for p in ps])
    for p in ps:
        p.before()
    gws.gws_adamw(packed, lr=3e-4, step=2)
    for p in ps:
        p.check(3e-4, 2, 0.9, 0.95, 1e-8)


def test_vectors_and_empty_tensors():
    f = lambda n, x=1.0: torch.full((n,), x, device=DEV)  # noqa: E731
    a = gws.AdamWTensor(p=f(33), g=f(33), m=f(33, 0.0), v=f(33, 0.0))
    e = gws.AdamWTensor(p=f(0), g=f(0), m=f(0), v=f(0))
    e2 = gws.AdamWTensor(p=f(0).view(0, 8), g=f(0).view(0, 8), m=f(0).view(0, 8), v=f(0).view(0, 8))
    gws.gws_adamw([e, a, e2], lr=0.5, step=1)
    # the first step moves by lr whatever the gradient's size
    assert torch.allclose(a.p, f(33, 0.5), atol=1e-6)
    gws.gws_adamw([], lr=0.5, step=1)
    gws.gws_adamw([e], lr=0.5, step=1)


def test_a_step_without_a_finite_gradient_norm_is_left_out():
    for bad in (math.nan, math.inf, -math.inf):
        ps = [Parameter(1, 5, 70, True), Parameter(2, 5, 70, False)]
        before = [w.clone() for p in ps for w in p.wholes]
        gws.gws_adamw([p.desc for p in ps], lr=1e-3, step=3, grad_scale=torch.tensor([bad], device=DEV))
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(before, (w for p in ps for w in p.wholes)))


@pytest.mark.parametrize("codes", [False, True])
def test_gradients_at_the_edge_of_the_numbers(codes):
    rows, cols = 8, 96
    rng = np.random.default_rng(3)
    g = (rng.standard_normal((rows, cols)) * 1e-3).astype(np.float32)
    g[0], g[1], g[2] = 0.0, 1e-30, 3e18
    g[3, 40], g[4, 70], g[5, 0] = math.nan, math.inf, -math.inf
    g[6, ::2] = 1e10                                              # a block of very different sizes
    z = np.zeros((rows, cols), dtype=np.float32)
    p = Parameter(4, rows, cols, codes, True, g=g, m=z, v=z)
    for step in (1, 2, 3):
        p.before()
        gws.gws_adamw([p.desc], lr=1e-3, step=step)
        p.check(1e-3, step, 0.9, 0.95, 1e-8)
    fine = [0, 1, 2, 6, 7]
    assert torch.isfinite(p.p[fine]).all()
    if codes:   # what shares a scale with a NaN becomes one, and nothing else
        assert torch.isfinite(p.p[3, :32]).all() and torch.isnan(p.p[3, 32:64]).all() and torch.isfinite(p.p[3, 64:]).all()
        assert torch.isfinite(p.p[5, 32:]).all()
    else:
        assert int((~torch.isfinite(p.p)).sum()) == 3


def test_scales_at_either_end():
    """Blocks whose largest magnitude is a power of two, 448 of one, the next number after it, and beyond the smallest and the largest scale."""
    tops = np.array([1.0, 448.0, np.nextafter(np.float32(448), np.float32(449)), 1.75 * 2.0 ** -100, 2.0 ** -120, 2.0 ** -140, 2.0 ** 100, 3.0e38], dtype=np.float32)
    rows = len(tops)
    g = np.tile(np.linspace(-1, 1, 64, dtype=np.float32), (rows, 1)) * tops[:, None]
    g[:, 0] = tops
    z = np.zeros_like(g)
    p = Parameter(5, rows, 64, True, True, g=g, m=z, v=z)
    p.before()
    gws.gws_adamw([p.desc], lr=1e-3, step=1, beta1=0.0, beta2=0.0)      # m = g, r = |g| where its square is a number
    p.check(1e-3, 1, 0.0, 0.0, 1e-8)


def test_rounding_at_random_keeps_the_mean():
    """m = g at 64 places between two neighbours, thousands of elements each: the share that goes up is the place, within five standard deviations."""
    rows, cols = 2048, 64
    place = np.arange(64) / 64.0
    g = np.tile((1.0 + place / 8).astype(np.float32), (rows, 1))
    g[:, [0, 32]] = 448.0                                              # the scale of both blocks is 1
    z = np.zeros_like(g)
    p = Parameter(6, rows, cols, True, True, g=g, m=z, v=z)
    gws.gws_adamw([p.desc], lr=0.0, step=1, beta1=0.0, beta2=0.0)
    for a in (p.m, p.v):
        v = ref.decode_state(a.codes.cpu().numpy(), a.xscale.cpu().numpy())
        up = (v == 1.125).mean(axis=0)
        assert set(np.unique(v)) <= {1.0, 1.125, 448.0}
        for c in range(64):
            if c not in (0, 32):
                assert abs(up[c] - place[c]) <= 5 * math.sqrt(place[c] * (1 - place[c]) / rows) + 2.0 ** -16, c


def test_a_slow_mean_moves():
    """With beta2 = 0.999 a step changes r by less than a hundredth of a spacing: over 400 steps it still follows the 64-bit mean."""
    rows, cols, steps = 64, 512, 400
    g = np.full((rows, cols), 0.5, dtype=np.float32)
    g[:, ::32] = 1.0
    z = np.zeros_like(g)
    p = Parameter(7, rows, cols, True, True, g=g, m=z, v=np.where(g == 1.0, 2.0, 1.0).astype(np.float32))
    packed = gws.pack_adamw([p.desc])
    for step in range(1, steps + 1):
        gws.gws_adamw(packed, lr=0.0, step=step, beta1=0.9, beta2=0.999)
    r = ref.decode_state(p.v.codes.cpu().numpy(), p.v.xscale.cpu().numpy())[:, 1::32]
    want = math.sqrt(0.999 ** steps + (1 - 0.999 ** steps) * 0.25)      # 0.869
    # Without rounding r goes to r' = sqrt(0.999 r^2 + 0.00025), from 1 to `want`.  A step's rounding is unbiased and adds s^2 f (1 - f) of variance, with spacing
    # s = 1/16 (r < 1) and place f = |r' - r| / s <= 0.006: 2.3e-5, after 400 steps at most 0.0092, a standard deviation of 0.096 of one element, 0.003 of the
    # mean of 1024.  The mean is moved by half of r''s curvature (0.00038) times that variance a step: 0.0007 in all.
    assert abs(r.mean() - want) <= 5 * 0.003 + 0.0007, (r.mean(), want)


@pytest.mark.parametrize("sizes", [[(1, 1)], [(1, 7), (33, 130)], [(300, 1000), (1, 5), (2, 16), (1000, 768)]])
def test_gradient_norm(sizes):
    ps = [Parameter(i, r, c, g_fp32=i % 2 == 0, ld=-(-c // 8) * 8 + 8) for i, (r, c) in enumerate(sizes)]
    packed = gws.pack_adamw([p.desc for p in ps])
    want = math.sqrt(sum(float((p.g.double() ** 2).sum()) for p in ps))
    ws, out = torch.full((gws.gws_grad_norm_workspace_bytes(packed) // 4,), math.nan, device=DEV), torch.zeros(2, device=DEV)
    for limit, factor in ((0.0, 1.0), (want * 0.25, 0.25), (want * 3, 1.0), (-1.0, 1.0)):
        gws.gws_grad_norm(packed, out, ws, max_norm=limit)
        assert abs(float(out[0]) - want) <= 2.0 ** -23 * want and abs(float(out[1]) - factor) <= 2.0 ** -23
    first = out.clone()
    gws.gws_grad_norm(packed, out, ws, max_norm=-1.0)
    assert torch.equal(first, out)
    for bad in (math.nan, math.inf):
        ps[-1].g[0, 0] = bad
        gws.gws_grad_norm(packed, out, ws, max_norm=1.0)
        assert torch.isnan(out).all()


def test_gradient_norm_of_many_of_nothing_and_of_small_numbers():
    out = torch.full((2,), 5.0, device=DEV)
    gws.gws_grad_norm([], out, None, max_norm=1.0)
    assert out.tolist() == [0.0, 1.0]
    g = torch.full((70, 64), 2.0 ** -100, device=DEV)                  # squares below fp32
    ts = [gws.AdamWTensor(p=g, g=g, m=g, v=g) for _ in range(500)]
    packed = gws.pack_adamw(ts)
    ws = torch.empty(gws.gws_grad_norm_workspace_bytes(packed), dtype=torch.uint8, device=DEV)
    gws.gws_grad_norm(packed, out, ws)
    assert abs(float(out[0]) / (2.0 ** -100 * math.sqrt(500 * 70 * 64)) - 1) <= 2.0 ** -23


def test_elements_past_32_bits():
    """A matrix whose last rows lie past 2^32 elements of its buffer."""
    rows, cols, ld = 33, 40, 1 << 27
    if torch.cuda.mem_get_info()[0] < 120 << 30:
        pytest.skip("no room")
    gen = torch.Generator(device=DEV).manual_seed(1)
    buf = lambda dtype: torch.empty(rows, ld, dtype=dtype, device=DEV)[:, :cols]  # noqa: E731
    p, g, m, v, w = buf(torch.float32), buf(torch.bfloat16), buf(torch.float32), buf(torch.float32), buf(torch.bfloat16)
    for t in (p, g, m, v):
        t.copy_(torch.randn(rows, cols, generator=gen, device=DEV))
    v.abs_()
    small = [t.clone() for t in (p, g, m, v, w)]
    gws.gws_adamw([gws.AdamWTensor(p=p, g=g, m=m, v=v, w=w)], lr=1e-2, step=3)
    gws.gws_adamw([gws.AdamWTensor(p=small[0], g=small[1], m=small[2], v=small[3], w=small[4])], lr=1e-2, step=3)
    assert all(torch.equal(a, b) for a, b in zip((p, m, v, w), (small[0], small[2], small[3], small[4])))


def test_more_groups_than_32_bits_count():
    """Half a billion rows of one column, whose blocks of 32 are more groups of four than 2^32; and a gradient of as many groups of eight."""
    if torch.cuda.mem_get_info()[0] < 120 << 30:
        pytest.skip("no room")
    rows = (1 << 29) + 1000
    z = lambda *s, dtype: torch.zeros(*s, dtype=dtype, device=DEV)  # noqa: E731
    p, g = z(rows, 8, dtype=torch.float32)[:, :1], z(rows, 8, dtype=torch.bfloat16)[:, :1]
    held = [gws.Act8(z(rows, 8, dtype=torch.uint8)[:, :1], z(rows, 1, dtype=torch.uint8)) for _ in range(2)]
    marks = [0, 1, 12345, (1 << 29) - 1, 1 << 29, rows - 1]
    for r in marks:
        g[r] = 1.0 + r % 7
    gws.gws_adamw([gws.AdamWTensor(p=p, g=g, m=held[0], v=held[1], seed=3)], lr=0.25, step=1)
    assert int((p != 0).sum()) == len(marks)
    assert all(abs(float(p[r]) + 0.25) < 1e-6 and int(held[0].codes[r]) != 0 and int(held[0].xscale[r]) != 127 for r in marks)
    assert int((held[1].codes != 0).sum()) == len(marks)
    del p, g, held
    torch.cuda.empty_cache()
    rows, cols = 1 << 15, (1 << 20) + 8
    g = z(rows, cols, dtype=torch.bfloat16)
    for r, c in ((0, 0), (7, cols - 1), (rows - 1, cols - 1), (rows // 2, 5)):
        g[r, c] = 2.0
    small = z(rows, 8, dtype=torch.float32)
    t = gws.pack_adamw([gws.AdamWTensor(p=small, g=small, m=small, v=small)])
    t.arr[0].g, t.arr[0].g_is_fp32, t.arr[0].cols, t.arr[0].ld = g.data_ptr(), 0, cols, cols       # of the fields the norm reads
    out, ws = z(2, dtype=torch.float32), torch.empty(gws.gws_grad_norm_workspace_bytes(t), dtype=torch.uint8, device=DEV)
    gws.gws_grad_norm(t, out, ws, max_norm=1.0)
    assert out.tolist() == [4.0, 0.25]
