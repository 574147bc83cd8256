"""The gated feed-forward block, forward and backward, against 64 bits.

Bounds, from the definition: a sum of K products in fp32, in any order, is within e = K 2^-24 sum |products| of the exact one; an output
rounded once to BF16 within 2^-9 of its size of that; and the gate's own arithmetic (a few fp32 operations, each within 2^-23 of its
size, the argument of exp within 2^-22 (1 + |w|)) adds less than 2^-16 (1 + |g|) of what it multiplies.  |a'| < 1.2 for both activations."""
import math

import pytest
import torch

import gated_ref as ref
import paper_2505_11170_amd as gws
from gpu_util import DEV, ensure_built

pytestmark = pytest.mark.gpu
ARITH = 2.0 ** -16


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_built()


def rand(seed, rows, cols, std=1.0, ld=None):
    """BF16 [rows x cols] in a buffer of `ld` columns whose others are NaN."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.full((rows, ld or cols), math.nan, dtype=torch.bfloat16, device=DEV)
    x[:, :cols] = (torch.randn(rows, cols, generator=gen, device=DEV) * std).bfloat16()
    return x[:, :cols]


def room(rows, cols, ld=None, dtype=torch.bfloat16):
    whole = torch.full((rows, ld or cols), 7, dtype=dtype, device=DEV)
    return whole[:, :cols], whole


def kept_buffers(kept, M, F, pad=0):
    """GatedSaved to be written, and its whole buffers."""
    if kept == "none":
        return None, []
    if kept == "bf16":
        (g, gw), (u, uw) = room(M, F, F + pad), room(M, F, F + 2 * pad)
        return gws.GatedSaved(g=g, u=u), [(gw, F), (uw, F)]
    parts = [room(M, n, n + p, torch.uint8) for n, p in ((F, pad), (F // 32, 3 if pad else 0), (F, 2 * pad), (F // 32, 5 if pad else 0))]
    return (gws.GatedSaved(g8=gws.Act8(parts[0][0], parts[1][0]), u8=gws.Act8(parts[2][0], parts[3][0])),
            [(w, n) for (_, w), n in zip(parts, (F, F // 32, F, F // 32))])


def kept_inputs(kept, g, u, pad=0):
    """GatedSaved that holds these BF16 G and U, and the values it stands for."""
    if kept == "bf16":
        return gws.GatedSaved(g=g, u=u), g.double(), u.double()
    out = []
    for v in (g, u):
        M, F = v.shape
        c, s = ref.encode(v.double())
        codes, scales = room(M, F, F + pad, torch.uint8)[0], room(M, F // 32, F // 32 + (3 if pad else 0), torch.uint8)[0]
        codes.copy_(c)
        scales.copy_(s)
        out.append(gws.Act8(codes, scales))
    return gws.GatedSaved(g8=out[0], u8=out[1]), ref.decode(out[0].codes, out[0].xscale), ref.decode(out[1].codes, out[1].xscale)


def check_fwd(M, K, F, nk, act, kept, pad=0, x=None, std=0.02, seed=0):
    x = rand(seed + 1, M, K, ld=K + pad) if x is None else x
    shape = (F, K) if nk else (K, F)
    wg, wu = (rand(seed + s, *shape, std, ld=shape[1] + pad) for s in (2, 3))
    h, hw = room(M, F, F + pad)
    saved, whole = kept_buffers(kept, M, F, pad)
    gws.gws_gated_fwd(x, wg, wu, h, act, saved=saved, w_is_nk=nk)
    torch.cuda.synchronize()
    (g, eg), (u, eu) = ref.product(x, wg, nk), ref.product(x, wu, nk)
    a, _ = ref.gate(act, g)
    ref.assert_within(h, a * u, ref.BF16 * (a * u).abs() + 1.2 * u.abs() * eg + a.abs() * eu + eg * eu * 1.2 + ARITH * (1 + g.abs()) * (g * u).abs() + 1e-30, "h")
    if kept == "bf16":
        for t, v, e, n in ((saved.g, g, eg, "g"), (saved.u, u, eu, "u")):
            ref.assert_within(t, v, ref.BF16 * v.abs() + e + 1e-30, n)
    elif kept == "e4m3":
        for t, v, e, n in ((saved.g8, g, eg, "g8"), (saved.u8, u, eu, "u8")):
            ref.assert_kept(t.codes, t.xscale, v, e, n)
    for w, n in [(hw, F)] + whole:
        assert (w[:, n:] == 7).all()     # past a row's data nothing is written


def check_bwd(M, D, F, nk, act, kept, pad=0, src="dy", h=True, seed=0, gstd=1.0):
    saved, g, u = kept_inputs(kept, rand(seed + 11, M, F, gstd), rand(seed + 12, M, F), pad)
    both, bw = room(M, 2 * F, 2 * F + pad)
    dg, du = both[:, :F], both[:, F:]           # two halves of one buffer
    hh, hw = room(M, F, F + pad)
    if src == "dy":
        dy = rand(seed + 13, M, D, 1e-3, ld=D + pad)
        shape = (D, F) if nk else (F, D)
        wd = rand(seed + 14, *shape, 0.02, ld=shape[1] + pad)
        gws.gws_gated_bwd(dy, wd, saved, dg, du, act, h=hh if h else None, w_is_nk=nk)
        dh, e = ref.product(dy, wd, not nk)
    else:
        d = rand(seed + 13, M, F, 1e-3, ld=F + pad)
        gws.gws_gated_bwd_h(d, saved, dg, du, act, h=hh if h else None)
        dh, e = d.double(), 0.0
    torch.cuda.synchronize()
    a, slope = ref.gate(act, g)
    arith = ARITH * (1 + g.abs())
    ref.assert_within(dg, dh * u * slope, ref.BF16 * (dh * u * slope).abs() + (u * slope).abs() * e + arith * (dh * u).abs() + 1e-38, "dg")
    ref.assert_within(du, dh * a, ref.BF16 * (dh * a).abs() + a.abs() * e + arith * (dh * g).abs() + 1e-38, "du")
    if h:
        ref.assert_within(hh, a * u, ref.BF16 * (a * u).abs() + arith * (g * u).abs() + 1e-38, "h")
    else:
        assert (hw == 7).all()
    assert (bw[:, 2 * F:] == 7).all() and (hw[:, F:] == 7).all()


def check_dx(M, K, F, nk, pad=0, seed=0):
    both = rand(seed + 21, M, 2 * F, 1e-3, ld=2 * F + pad)
    dg, du = both[:, :F], both[:, F:]
    shape = (F, K) if nk else (K, F)
    wg, wu = (rand(seed + s, *shape, 0.02, ld=shape[1] + pad) for s in (22, 23))
    dx, whole = room(M, K, K + pad)
    gws.gws_gated_bwd_x(dg, du, wg, wu, dx, w_is_nk=nk)
    torch.cuda.synchronize()
    (p, _), (q, _) = ref.product(dg, wg, not nk), ref.product(du, wu, not nk)
    _, e = ref.product(torch.cat([dg, du], 1), torch.cat([wg if nk else wg.t(), wu if nk else wu.t()], 0), False)
    ref.assert_within(dx, p + q, ref.BF16 * (p + q).abs() + e + 1e-38, "dx")
    assert (whole[:, K:] == 7).all()


SIZES = [(1, 32, 32), (1, 2048, 5632), (3, 96, 64), (15, 768, 2048), (16, 64, 96), (17, 160, 32), (63, 128, 224), (64, 256, 256), (65, 2048, 352),
         (128, 64, 128), (200, 96, 544), (257, 320, 160), (512, 512, 512), (1021, 768, 2048), (1300, 416, 1376)]


@pytest.mark.parametrize("kept", ["none", "bf16", "e4m3"])
@pytest.mark.parametrize("nk", [False, True])
@pytest.mark.parametrize("M,K,F", SIZES)
def test_forward(M, K, F, nk, kept):
    check_fwd(M, K, F, nk, (M + F // 32) % 2, kept, pad=0 if M % 2 else 40)


@pytest.mark.parametrize("kept", ["bf16", "e4m3"])
@pytest.mark.parametrize("nk", [False, True])
@pytest.mark.parametrize("M,D,F", SIZES)
def test_backward_from_dy(M, D, F, nk, kept):
    check_bwd(M, D, F, nk, (M + F // 32) % 2, kept, pad=0 if M % 2 else 40, h=M % 3 != 0)


@pytest.mark.parametrize("kept", ["bf16", "e4m3"])
@pytest.mark.parametrize("M,F", [(1, 32), (5, 96), (77, 5632), (1021, 2048)])
def test_backward_from_dh(M, F, kept):
    check_bwd(M, 0, F, False, M % 2, kept, pad=0 if M % 2 else 40, src="dh", h=M != 77)


@pytest.mark.parametrize("nk", [False, True])
@pytest.mark.parametrize("M,K,F", SIZES)
def test_input_gradient(M, K, F, nk):
    check_dx(M, K, F, nk, pad=0 if M % 2 else 40)


@pytest.mark.parametrize("nk", [False, True])
def test_whole_tiles_of_a_training_batch(nk):
    check_fwd(2048, 512, 1536, nk, ref.SILU, "e4m3")
    check_bwd(2048, 512, 1536, nk, ref.GELU, "e4m3")
    check_bwd(2048, 512, 1536, nk, ref.SILU, "bf16")
    check_dx(2048, 512, 1536, nk)


@pytest.mark.parametrize("act", [ref.SILU, ref.GELU])
def test_gate_over_its_whole_range(act):
    # G of every size that BF16 has, both signs, U and dH one: where exp overflows, where q is 0 or 1, at zero
    g = torch.cat([torch.linspace(-40, 40, 4096), torch.tensor([0.0, -0.0, 1e-30, -1e-30, 88.0, -88.0, 89.0, -89.0, 104.0, -104.0, 1e4, -1e4, 1e20, -1e20,
                                                                 3e38, -3e38])]).bfloat16().to(DEV)
    g = torch.cat([g, g.new_zeros(-g.numel() % 32)]).reshape(1, -1)
    one = torch.ones_like(g)
    for kept in ("bf16", "e4m3"):
        saved, gv, uv = kept_inputs(kept, g, one)
        dg, du, h = (torch.zeros_like(g) for _ in range(3))
        gws.gws_gated_bwd_h(one, saved, dg, du, act, h=h)
        torch.cuda.synchronize()
        a, slope = ref.gate(act, gv.clamp(-1e30, 1e30))      # the 64-bit formula's own g^3 overflows beyond
        a, slope = torch.where(gv > 1e20, gv, a), torch.where(gv.abs() > 1e20, (gv > 0).double(), slope)
        a, slope = torch.nan_to_num(a), torch.where(torch.isnan(slope), (gv > 0).double(), slope)
        tol = ref.BF16 * a.abs() + ARITH * (1 + gv.abs()) * (gv.abs() < 200) + 1e-30
        ref.assert_within(du, a, tol, "du")
        ref.assert_within(h, a, tol, "h")
        ref.assert_within(dg, slope, ref.BF16 * slope.abs() + ARITH * (1 + gv.abs().clamp(max=200)), "dg")


def test_rows_do_not_meet():
    # a token of NaN, one of infinities and one of zeros: every other row has the bits it has without them
    M, K, F = 300, 256, 512
    x = rand(1, M, K).contiguous()
    bad = x.clone()
    bad[7], bad[130], bad[299] = math.nan, math.inf, 0.0
    others = [r for r in range(M) if r not in (7, 130, 299)]
    wg, wu = rand(2, F, K, 0.02), rand(3, F, K, 0.02)
    out = []
    for v in (x, bad):
        h = torch.zeros(M, F, dtype=torch.bfloat16, device=DEV)
        saved, _ = kept_buffers("e4m3", M, F)
        gws.gws_gated_fwd(v, wg, wu, h, saved=saved, w_is_nk=True)
        torch.cuda.synchronize()
        out.append((h, saved))
    (h0, s0), (h1, s1) = out
    assert torch.equal(h0[others], h1[others])
    for p, q in ((s0.g8, s1.g8), (s0.u8, s1.u8)):
        assert torch.equal(p.codes[others], q.codes[others]) and torch.equal(p.xscale[others], q.xscale[others])
        assert (q.xscale[7] == 255).all() and (q.codes[7] == 127).all() and (q.xscale[299] == 127).all() and ((q.codes[299] & 127) == 0).all()
    assert torch.isnan(h1[7]).all() and (h1[299] == 0).all()
    # and backward: a NaN block of a kept G reaches its own 32 columns of dG, dU and H only
    dg, du, hh = (torch.zeros(M, F, dtype=torch.bfloat16, device=DEV) for _ in range(3))
    s0.g8.xscale[11, 3] = 255
    gws.gws_gated_bwd(rand(4, M, K, 1e-3), rand(5, F, K, 0.02), s0, dg, du, h=hh)
    torch.cuda.synchronize()
    want = torch.zeros(M, F, dtype=torch.bool, device=DEV)
    want[11, 96:128] = True
    for t in (dg, du, hh):
        assert torch.equal(torch.isnan(t), want)


def test_results_in_the_place_of_what_they_are_formed_from():
    M, D, F = 333, 128, 480
    g, u, dy, wd = rand(1, M, F).contiguous(), rand(2, M, F).contiguous(), rand(3, M, D, 1e-3), rand(4, F, D, 0.02)
    dh = rand(5, M, F, 1e-3).contiguous()
    for from_dy in (True, False):
        outs = [torch.zeros(M, F, dtype=torch.bfloat16, device=DEV) for _ in range(3)]
        if from_dy:
            gws.gws_gated_bwd(dy, wd, gws.GatedSaved(g=g, u=u), outs[0], outs[1], h=outs[2])
        else:
            gws.gws_gated_bwd_h(dh, gws.GatedSaved(g=g, u=u), outs[0], outs[1], h=outs[2])
        g1, u1, d1, h1 = g.clone(), u.clone(), dh.clone(), torch.zeros_like(g)
        if from_dy:
            gws.gws_gated_bwd(dy, wd, gws.GatedSaved(g=g1, u=u1), u1, g1, h=h1)
            got = (u1, g1, h1)
        else:
            gws.gws_gated_bwd_h(d1, gws.GatedSaved(g=g1, u=u1), g1, d1, h=u1)
            got = (g1, d1, u1)
        torch.cuda.synchronize()
        for a, b in zip(outs, got):
            assert torch.equal(a, b)


def test_offsets_beyond_32_bits():
    M, K, F, ld = 70000, 32, 32, 32768
    x = rand(1, M, K)
    wg, wu = rand(2, F, K, 0.1), rand(3, F, K, 0.1)
    far = torch.empty(M, ld, dtype=torch.bfloat16, device=DEV)
    near = torch.zeros(M, F, dtype=torch.bfloat16, device=DEV)
    gws.gws_gated_fwd(x, wg, wu, near, w_is_nk=True)
    gws.gws_gated_fwd(x, wg, wu, far[:, :F], saved=gws.GatedSaved(g=far[:, 64:96], u=far[:, 96:128]), w_is_nk=True)
    torch.cuda.synchronize()
    assert torch.equal(far[:, :F], near)
    dg, du, h = (torch.zeros_like(near) for _ in range(3))
    for from_h in (False, True):
        dy = rand(4, M, K, 1e-3)
        g, u = far[:, 64:96].contiguous(), far[:, 96:128].contiguous()
        if from_h:
            gws.gws_gated_bwd_h(dy, gws.GatedSaved(g=g, u=u), dg, du, h=h)
            gws.gws_gated_bwd_h(dy, gws.GatedSaved(g=far[:, 64:96], u=far[:, 96:128]), far[:, 128:160], far[:, 160:192], h=far[:, 192:224])
        else:
            gws.gws_gated_bwd(dy, wg, gws.GatedSaved(g=g, u=u), dg, du, h=h)
            gws.gws_gated_bwd(dy, wg, gws.GatedSaved(g=far[:, 64:96], u=far[:, 96:128]), far[:, 128:160], far[:, 160:192], h=far[:, 192:224])
        torch.cuda.synchronize()
        assert torch.equal(far[:, 128:160], dg) and torch.equal(far[:, 160:192], du) and torch.equal(far[:, 192:224], h)
    dx = torch.zeros(M, K, dtype=torch.bfloat16, device=DEV)
    gws.gws_gated_bwd_x(dg, du, wg, wu, dx, w_is_nk=True)
    gws.gws_gated_bwd_x(far[:, 128:160], far[:, 160:192], wg, wu, far[:, 256:288], w_is_nk=True)
    torch.cuda.synchronize()
    assert torch.equal(far[:, 256:288], dx)


def test_the_same_call_gives_the_same_bits():
    M, K, F = 700, 768, 1024
    x, wg, wu = rand(1, M, K), rand(2, K, F, 0.02), rand(3, K, F, 0.02)
    outs = []
    for _ in range(2):
        h = torch.zeros(M, F, dtype=torch.bfloat16, device=DEV)
        s = gws.GatedSaved(g=torch.zeros_like(h), u=torch.zeros_like(h))
        gws.gws_gated_fwd(x, wg, wu, h, saved=s)
        torch.cuda.synchronize()
        outs.append((h, s.g, s.u))
    assert all(torch.equal(a, b) for a, b in zip(*outs))


def test_captured_in_a_graph_and_replayed():
    M, K, F = 130, 256, 512
    x, wg, wu, wd = rand(1, M, K), rand(2, F, K, 0.02), rand(3, F, K, 0.02), rand(4, K, F, 0.02)
    dy = rand(5, M, K, 1e-3)
    bufs = {k: torch.zeros(M, F, dtype=torch.bfloat16, device=DEV) for k in ("h", "dg", "du", "h2")}
    dx = torch.zeros(M, K, dtype=torch.bfloat16, device=DEV)
    saved, _ = kept_buffers("e4m3", M, F)

    def step():
        gws.gws_gated_fwd(x, wg, wu, bufs["h"], saved=saved, w_is_nk=True)
        gws.gws_gated_bwd(dy, wd, saved, bufs["dg"], bufs["du"], h=bufs["h2"], w_is_nk=True)
        gws.gws_gated_bwd_x(bufs["dg"], bufs["du"], wg, wu, dx, w_is_nk=True)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (31, 32, 33):
        x.copy_(rand(seed, M, K))
        dy.copy_(rand(seed + 10, M, K, 1e-3))
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in (*bufs.values(), dx, saved.g8.codes, saved.u8.xscale)]
        for t in (*bufs.values(), dx):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, (*bufs.values(), dx, saved.g8.codes, saved.u8.xscale)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("act", [ref.SILU, ref.GELU])
@pytest.mark.parametrize("nk", [False, True])
def test_gradient_against_differences(act, nk):
    # L = sum(C .* Y), Y = (a(X Wg) .* (X Wu)) Wd: dX along a direction against the difference quotient of the 64-bit block
    M, K, F = 48, 128, 256
    shape, dshape = ((F, K), (K, F)) if nk else ((K, F), (F, K))
    x, wg, wu, wd, c = rand(1, M, K), rand(2, *shape, 0.09), rand(3, *shape, 0.09), rand(4, *dshape, 0.06), rand(5, M, K)
    h = torch.zeros(M, F, dtype=torch.bfloat16, device=DEV)
    saved, _ = kept_buffers("bf16", M, F)
    gws.gws_gated_fwd(x, wg, wu, h, act, saved=saved, w_is_nk=nk)
    dg, du = torch.zeros_like(h), torch.zeros_like(h)
    dx = torch.zeros(M, K, dtype=torch.bfloat16, device=DEV)
    gws.gws_gated_bwd(c, wd, saved, dg, du, act, w_is_nk=nk)
    gws.gws_gated_bwd_x(dg, du, wg, wu, dx, w_is_nk=nk)
    torch.cuda.synchronize()

    def loss(v):
        g, u = (v @ (w.double().t() if nk else w.double()) for w in (wg, wu))
        y = (ref.gate(act, g)[0] * u) @ (wd.double().t() if nk else wd.double())
        return (c.double() * y).sum(dim=1)

    for seed in (6, 7):
        v = rand(seed, M, K).double()
        eps = 2.0 ** -12
        slope = (loss(x.double() + eps * v) - loss(x.double() - eps * v)) / (2 * eps)
        # every rounding on the way (G, U, dG, dU, dX) is within 2^-9 of its own size; a' changes by less than the rounding of G
        # times |g a''| < 1.2: together below 5 roundings of what is summed, taken without signs
        g, u = (x.double() @ (w.double().t() if nk else w.double()) for w in (wg, wu))
        dh = c.double() @ (wd.double() if nk else wd.double().t())
        a, s = ref.gate(act, g)
        tg, tu = (dh * u).abs() * 1.2, (dh * a).abs() + (dh * g).abs() * 0.5
        wga, wua = (w.double().abs() if nk else w.double().abs().t() for w in (wg, wu))
        tol = 5 * 2.0 ** -9 * ((tg @ wga + tu @ wua) * v.abs()).sum(dim=1)
        ref.assert_within((dx.double() * v).sum(dim=1), slope, tol, "slope")
        assert (slope.abs() > 0).all() and tol.median() < slope.abs().max()
