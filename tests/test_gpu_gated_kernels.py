"""Every kernel and tile behind the gated block's entry points, at sizes that take it: whole tiles, edges of rows and columns, half a K-step
of 64 at the end of the contraction (of either product of the input gradient), one K-step, and activations whose scale saturates."""
import ctypes

import pytest
import torch

import gated_ref as ref
import paper_2505_11170_amd as gws
from gpu_util import DEV, ensure_built
from paper_2505_11170_amd import binding
from test_gpu_gated import check_bwd, check_dx, check_fwd, kept_buffers, rand

pytestmark = pytest.mark.gpu
ANY, STREAM, MIDDLE, LARGE, SHARED = (1, 0, 0), 2, (3, 0, 0), (4, 0, 0), (5, 0, 0)
KEPT = {"none": 0, "bf16": 1, "e4m3": 2}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_built()


def taken(form, *args, **kw):
    assert gws.gws_gated_form(*args, **kw) == form, (gws.gws_gated_form(*args, **kw), args, kw)


# M, K, F, kernel; of the tiles of few tokens 16-column tiles of both weights together, narrow ones where the layout and what is kept allow them
FORWARD = [(5, 32, 160, ANY), (7, 96, 96, (STREAM, 1, 2)), (9, 64, 64, (STREAM, 1, 2)), (3, 96, 4640, (STREAM, 1, 4)), (14, 160, 4704, (STREAM, 1, 4)),
           (19, 96, 96, (STREAM, 2, 4)), (32, 1024, 128, (STREAM, 2, 4)), (239, 480, 1088, (STREAM, 4, 4)), (64, 512, 5632, (STREAM, 4, 4)),
           (84, 96, 4960, (STREAM, 8, 4)), (128, 256, 5632, (STREAM, 8, 4)), (700, 736, 2080, MIDDLE), (1024, 64, 2048, MIDDLE), (256, 2048, 5632, MIDDLE),
           (408, 96, 4160, SHARED), (914, 352, 3520, SHARED),
           (1300, 96, 5024, SHARED), (1792, 384, 2816, SHARED), (1460, 288, 4448, SHARED),
           (1024, 896, 5632, LARGE), (2091, 736, 1952, LARGE), (1211, 768, 3296, LARGE), (2304, 2048, 3584, LARGE)]
BACKWARD = [(5, 32, 160, ANY), (7, 96, 96, (STREAM, 1, 2)), (16, 64, 96, (STREAM, 1, 2)), (3, 96, 9248, (STREAM, 1, 4)), (13, 64, 12288, (STREAM, 1, 4)),
            (19, 96, 96, (STREAM, 2, 4)), (32, 1024, 128, (STREAM, 2, 4)), (202, 96, 2400, (STREAM, 4, 4)), (118, 448, 4800, (STREAM, 4, 4)),
            (1110, 96, 928, (STREAM, 8, 4)), (1021, 768, 2048, (STREAM, 8, 4)), (1211, 416, 2112, MIDDLE), (2048, 512, 2048, MIDDLE), (600, 1056, 5536, MIDDLE),
            (900, 96, 4288, SHARED), (1849, 224, 4768, SHARED), (4096, 768, 2048, SHARED), (2048, 2048, 5632, SHARED),
            (2560, 1152, 5632, LARGE), (2977, 864, 5248, LARGE), (2300, 2080, 5152, LARGE)]
GRADIENT = [(5, 160, 32, ANY), (7, 96, 96, (STREAM, 1, 2)), (16, 4160, 64, (STREAM, 1, 2)), (11, 12288, 96, (STREAM, 1, 4)), (21, 96, 96, (STREAM, 2, 2)),
            (32, 1024, 1024, (STREAM, 2, 2)), (184, 1376, 96, (STREAM, 2, 4)), (700, 768, 2016, (STREAM, 4, 4)), (701, 928, 96, (STREAM, 4, 4)),
            (955, 544, 160, (STREAM, 4, 4)), (584, 1696, 544, (STREAM, 8, 4)), (849, 1184, 544, (STREAM, 8, 4)), (2061, 480, 96, MIDDLE), (1169, 1696, 96, MIDDLE), (2048, 2048, 544, MIDDLE), (4096, 768, 1056, MIDDLE), (6000, 2016, 480, LARGE), (8192, 2048, 256, LARGE)]
# M, K, F, (kernel of the first launch, of the second, whether they share the rows rather than the columns)
FORWARD_SPLIT = [(2217, 1152, 3808, (LARGE, 2, False)), (1796, 1184, 4416, (LARGE, 2, True)), (1951, 1152, 4864, (LARGE, 3, False)),
                 (1820, 1120, 5056, (LARGE, 3, True)), (1927, 1280, 5152, (LARGE, 5, False)), (2914, 1376, 3424, (LARGE, 5, True))]
BACKWARD_SPLIT = [(5271, 1664, 3104, (LARGE, 2, False)), (3848, 1504, 4352, (LARGE, 2, True)), (3999, 1792, 5056, (LARGE, 3, False)),
                  (3814, 1824, 5280, (LARGE, 3, True))]
GRADIENT_SPLIT = [(2208, 1888, 672, (MIDDLE, 2, False)), (3289, 1280, 800, (MIDDLE, 2, True))]


@pytest.mark.parametrize("kept", ["none", "bf16", "e4m3"])
@pytest.mark.parametrize("nk", [False, True])
@pytest.mark.parametrize("M,K,F,forms", FORWARD_SPLIT)
def test_forward_of_two_launches(M, K, F, forms, nk, kept):
    assert gws.gws_gated_forms(gws.GATED_FWD, M, K, F, nk, KEPT[kept]) == forms
    check_fwd(M, K, F, nk, M % 2, kept, pad=8 * (M % 3))


@pytest.mark.parametrize("kept", ["bf16", "e4m3"])
@pytest.mark.parametrize("nk", [False, True])
@pytest.mark.parametrize("M,D,F,forms", BACKWARD_SPLIT)
def test_backward_of_two_launches(M, D, F, forms, nk, kept):
    assert gws.gws_gated_forms(gws.GATED_BWD, M, D, F, nk, KEPT[kept]) == forms
    check_bwd(M, D, F, nk, M % 2, kept, pad=8 * (M % 3))


@pytest.mark.parametrize("nk", [False, True])
@pytest.mark.parametrize("M,K,F,forms", GRADIENT_SPLIT)
def test_input_gradient_of_two_launches(M, K, F, forms, nk):
    assert gws.gws_gated_forms(gws.GATED_BWD_X, M, K, F, nk) == forms
    check_dx(M, K, F, nk, pad=8 * (M % 3))


# What check_dx runs: dG and dU are the halves of one buffer, and rows that start off the lines of 128 bytes count in the choice.
# M, K, F, w_is_nk or None for either, (kernel of the first launch, of the second, whether they share the rows)
GRADIENT_AS_RUN = [(849, 1184, 544, None, (MIDDLE, 0, False)), (584, 1696, 544, None, ((STREAM, 8, 4), 0, False)), (2061, 480, 96, None, (MIDDLE, 0, False)),
                   (3848, 1056, 608, None, (MIDDLE, 2, False)), (3943, 1056, 608, None, (MIDDLE, 2, False)), (4604, 928, 608, None, (MIDDLE, 2, False)),
                   (2478, 1632, 672, True, (MIDDLE, 2, False)), (2208, 1888, 672, False, (MIDDLE, 2, False)), (2208, 1888, 672, True, (MIDDLE, 0, False)),
                   (2692, 1536, 608, None, (MIDDLE, 2, True)), (3343, 1248, 608, None, (MIDDLE, 2, True)), (2051, 2016, 672, None, (MIDDLE, 2, True))]


@pytest.mark.parametrize("M,K,F,nk,forms", [(M, K, F, nk, forms) for M, K, F, one, forms in GRADIENT_AS_RUN for nk in ([False, True] if one is None else [one])])
def test_input_gradient_as_it_is_run(M, K, F, nk, forms):
    pad = 8 * (M % 3)
    assert gws.gws_gated_forms(gws.GATED_BWD_X, M, K, F, nk, lda=2 * F + pad, ldw=(K if nk else F) + pad) == forms
    check_dx(M, K, F, nk, pad=pad)


@pytest.mark.parametrize("nk", [False, True])
@pytest.mark.parametrize("M,K,F", [(8192, 2048, 64), (8192, 2048, 96), (6007, 2016, 160), (8190, 2048, 224), (8192, 2048, 288), (8191, 2048, 352), (8192, 2016, 416)])
def test_input_gradient_of_few_steps_in_large_tiles(M, K, F, nk):
    # the first product's half step of 64 in each place of the ring of K-steps, inside the unrolled six and behind them
    pad = 8 * (M % 3)
    assert gws.gws_gated_forms(gws.GATED_BWD_X, M, K, F, nk, lda=2 * F + pad, ldw=(K if nk else F) + pad) == (LARGE, 0, False)
    check_dx(M, K, F, nk, pad=pad)


@pytest.mark.parametrize("kept", ["bf16", "e4m3"])
@pytest.mark.parametrize("M,K,F,form", [(7, 96, 96, STREAM), (128, 256, 5632, STREAM), (700, 736, 2080, MIDDLE), (1300, 96, 5024, SHARED), (2091, 736, 1952, LARGE),
                                        (8192, 2048, 5632, LARGE), (2217, 1152, 3808, LARGE)])
def test_every_call_gives_the_same_bits(M, K, F, form, kept):
    # the forward call repeated, another one between, without a wait: what is kept (in 8 bits: codes that a last bit of a sum decides among them) and H
    f = gws.gws_gated_form(gws.GATED_FWD, M, K, F, True, KEPT[kept])
    assert f == form or f[0] == form
    gen = torch.Generator(device=DEV).manual_seed(M)
    def some(r, c, std):
        return (torch.randn(r, c, device=DEV, generator=gen) * std).bfloat16()
    x, other, wg, wu = some(M, K, 1.0), some(M, K, 1.0), some(F, K, 0.02), some(F, K, 0.02)
    h = torch.zeros(M, F, dtype=torch.bfloat16, device=DEV)
    saved, _ = kept_buffers(kept, M, F)
    outs = [h] + ([saved.g, saved.u] if kept == "bf16" else [saved.g8.codes, saved.g8.xscale, saved.u8.codes, saved.u8.xscale])
    gws.gws_gated_fwd(x, wg, wu, h, saved=saved, w_is_nk=True)
    want = [t.clone() for t in outs]
    for _ in range(4):
        for v in (other, x, other, x):
            gws.gws_gated_fwd(v, wg, wu, h, saved=saved, w_is_nk=True)
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


@pytest.mark.parametrize("kept", ["none", "bf16", "e4m3"])
@pytest.mark.parametrize("M,K,F,form", [(16384, 64, 5632, SHARED), (46007, 64, 2016, SHARED), (16384, 512, 5632, LARGE), (12211, 1024, 7520, LARGE)])
def test_forward_past_the_caches(M, K, F, form, kept):
    nk = M % 2 == 0
    assert gws.gws_gated_past_caches(gws.GATED_FWD, M, K, F, nk, KEPT[kept])
    taken(form, gws.GATED_FWD, M, K, F, nk, KEPT[kept])
    check_fwd(M, K, F, nk, M % 2, kept, pad=8 * (M % 3))


def test_two_launches_in_place():
    # dG and dU in the places of the kept BF16 values: each launch reads and writes its own columns, or rows, alone
    for M, D, F, forms in BACKWARD_SPLIT[:2]:
        assert gws.gws_gated_forms(gws.GATED_BWD, M, D, F, True, KEPT["bf16"]) == forms
        gen = torch.Generator(device=DEV).manual_seed(M)
        def some(r, c, std):
            return (torch.randn(r, c, device=DEV, generator=gen) * std).bfloat16()
        dy, w, g, u = some(M, D, 1e-3), some(D, F, 0.02), some(M, F, 1.0), some(M, F, 1.0)
        dg, du = torch.empty_like(g), torch.empty_like(u)
        gws.gws_gated_bwd(dy, w, gws.GatedSaved(g=g, u=u), dg, du, w_is_nk=True)
        gws.gws_gated_bwd(dy, w, gws.GatedSaved(g=g, u=u), g, u, w_is_nk=True)
        torch.cuda.synchronize()
        assert torch.equal(g, dg) and torch.equal(u, du)


@pytest.mark.parametrize("kept", ["none", "bf16", "e4m3"])
@pytest.mark.parametrize("nk", [False, True])
@pytest.mark.parametrize("M,K,F,form", FORWARD)
def test_forward(M, K, F, form, nk, kept):
    f = gws.gws_gated_form(gws.GATED_FWD, M, K, F, nk, KEPT[kept])
    if form == (STREAM, 1, 2) and (not nk or kept == "e4m3"):
        form = (STREAM, 1, 4)                        # 32 columns of each weight at least
    if form == (STREAM, 1, 4) and nk and kept != "e4m3":
        assert f in ((STREAM, 1, 2), (STREAM, 1, 4))
    else:
        taken(form, gws.GATED_FWD, M, K, F, nk, KEPT[kept])
    check_fwd(M, K, F, nk, M % 2, kept, pad=8 * (M % 3))


@pytest.mark.parametrize("kept", ["bf16", "e4m3"])
@pytest.mark.parametrize("nk", [False, True])
@pytest.mark.parametrize("M,D,F,form", BACKWARD)
def test_backward(M, D, F, form, nk, kept):
    taken(form, gws.GATED_BWD, M, D, F, nk, KEPT[kept])
    check_bwd(M, D, F, nk, M % 2, kept, pad=8 * (M % 3), h=M % 5 != 0)


@pytest.mark.parametrize("nk", [False, True])
@pytest.mark.parametrize("M,K,F,form", GRADIENT)
def test_input_gradient(M, K, F, form, nk):
    if form == (STREAM, 1, 2) and not nk and K < 4160:
        form = (STREAM, 1, 1)                        # 16 columns of a weight along the contraction
    if form == (STREAM, 4, 4) and not nk and K in (544, 768, 928):
        form = (STREAM, 4, 3)                        # 48 columns of one, where that leaves fewer compute units idle
    taken(form, gws.GATED_BWD_X, M, K, F, nk)
    check_dx(M, K, F, nk, pad=8 * (M % 3))


@pytest.mark.parametrize("M,F,form", [(9, 160, (STREAM, 1, 4)), (700, 2080, MIDDLE), (1300, 5024, SHARED), (2091, 1952, LARGE), (5, 160, ANY)])
def test_values_beyond_the_largest_scale(M, F, form):
    # one product per sum: G of up to 3.2e38, which its BF16 rounding and 464 2^119 = 3.08e38 lie below
    K = {ANY: 32, LARGE: 736}.get(form, 96)
    taken(form, gws.GATED_FWD, M, K, F, True, 2)
    x = torch.zeros(M, K, dtype=torch.bfloat16, device=DEV)
    x[:, 0] = torch.tensor([2.0 ** 64, -(2.0 ** 64), 2.0 ** 60, 1.0], dtype=torch.bfloat16).repeat(-(-M // 4))[:M].to(DEV)
    w = torch.zeros(F, K, dtype=torch.bfloat16, device=DEV)
    w[:, 0] = (2.0 ** 63 * (1.0 + torch.arange(F, device=DEV) % 32 * (0.875 / 31))).bfloat16()
    u = torch.zeros_like(w)
    h = torch.zeros(M, F, dtype=torch.bfloat16, device=DEV)
    saved, _ = kept_buffers("e4m3", M, F)
    gws.gws_gated_fwd(x, w, u, h, saved=saved, w_is_nk=True)
    torch.cuda.synchronize()
    codes, scales = ref.encode(x.double() @ w.double().t())
    assert int(scales.max()) == 246
    assert torch.equal(saved.g8.codes, codes) and torch.equal(saved.g8.xscale, scales)
    assert (saved.u8.codes & 127 == 0).all() and (saved.u8.xscale == 127).all()


@pytest.mark.parametrize("M,D,F", [(1021, 2048, 768), (2048, 256, 2048)])
def test_the_leading_dimension_of_an_h_that_is_left_out_says_nothing(M, D, F):
    lib, stream = binding.load_library(), torch.cuda.current_stream().cuda_stream
    dy, wd, g, u = rand(1, M, D), rand(2, F, D, 0.05), rand(3, M, F), rand(4, M, F)
    saved = binding._CGatedSaved(g.data_ptr(), u.data_ptr(), F, F)
    first = None
    for ldh in (0, -1, 1 << 30):
        dg, du = torch.zeros_like(g), torch.zeros_like(u)
        assert lib.gws_gated_bwd(dy.data_ptr(), M, D, D, wd.data_ptr(), F, D, 0, gws.ACT_SILU, ctypes.byref(saved), dg.data_ptr(), du.data_ptr(), F, None, ldh, stream) == 0
        first = first or (dg, du)
        assert torch.equal(first[0], dg) and torch.equal(first[1], du), ldh
