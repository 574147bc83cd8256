"""The tiles of the gated block with operands, kept values and results that lie more than 4 GiB apart, and with the widest rows that each takes:
the bits of the same call on matrices without gaps.  (tests/test_gpu_gated.py has the kernel of any size.)"""
import pytest
import torch

import paper_2505_11170_amd as gws
from gpu_util import DEV, ensure_built

pytestmark = pytest.mark.gpu
STREAM, MIDDLE, LARGE, SHARED = 2, 3, 4, 5
FOUR_GIB = 1 << 32


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_built()


@pytest.fixture(autouse=True)
def _memory():
    yield
    torch.cuda.empty_cache()   # up to 57 GB a case, of other sizes each


def beyond(rows, size, limit=1 << 28):
    """A leading dimension, on lines of 128 bytes, with which the last row starts past 4 GiB; `limit`: no wider rows than that."""
    return min(-(-FOUR_GIB // (size * (rows - 1) * 64)) * 64 + 64, limit - 64)


class Apart:
    """Matrices side by side in one buffer of rows of `ld`, whatever lies between."""

    def __init__(self, rows, ld, dtype=torch.bfloat16):
        self.buf, self.at = torch.empty(rows, ld, dtype=dtype, device=DEV), 0

    def room(self, cols):
        self.at += cols + (-cols % 64)
        assert self.at <= self.buf.shape[1]
        return self.buf[:, self.at - cols - (-cols % 64):][:, :cols]

    def put(self, t):
        r = self.room(t.shape[1])
        r.copy_(t)
        return r


def some(seed, rows, cols, std):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(rows, cols, device=DEV, generator=gen) * std).bfloat16()


def kept_near(kept, M, F, values=None):
    """G and U without gaps: room for them, or holding `values`."""
    if kept == "none":
        return None
    if kept == "bf16":
        return gws.GatedSaved(*(values or [torch.zeros(M, F, dtype=torch.bfloat16, device=DEV) for _ in range(2)]))
    a = [gws.Act8(torch.zeros(M, F, dtype=torch.uint8, device=DEV), torch.zeros(M, F // 32, dtype=torch.uint8, device=DEV)) for _ in range(2)]
    for t, v in zip(a, values or ()):
        gws.gws_act8_encode(v, t)
    return gws.GatedSaved(g8=a[0], u8=a[1])


def kept_far(kept, near, results, fill):
    """The same in `results` or, codes and scales, in a buffer of bytes of their own."""
    place = (lambda b, t: b.put(t)) if fill else (lambda b, t: b.room(t.shape[1]))
    if kept == "none":
        return None, []
    if kept == "bf16":
        s = gws.GatedSaved(g=place(results, near.g), u=place(results, near.u))
        return s, [s.g, s.u]
    M = near.g8.codes.shape[0]
    bytes_ = Apart(M, beyond(M, 1), torch.uint8)
    a = [gws.Act8(place(bytes_, t.codes), place(bytes_, t.xscale)) for t in (near.g8, near.u8)]
    return gws.GatedSaved(g8=a[0], u8=a[1]), [t for v in a for t in (v.codes, v.xscale)]


def parts(kept, s):
    return [] if kept == "none" else [s.g, s.u] if kept == "bf16" else [s.g8.codes, s.g8.xscale, s.u8.codes, s.u8.xscale]


def assert_form(form, op, M, K, F, nk, kept, *strides):
    for lda, ldw in strides:
        first, second, by_rows = gws.gws_gated_forms(op, M, K, F, nk, {"none": 0, "bf16": 1, "e4m3": 2}[kept], lda=lda, ldw=ldw)
        assert ((first[0], second, by_rows) if second else first[0]) == form, (first, second, by_rows)


# M, K, F, [F x K], kernel, rows of X and of the weights: None past 4 GiB, else that many elements (the widest a kernel takes is 8 below its limit)
LD128, LD256 = (1 << 24) - 8, (1 << 23) - 8
FORWARD = [(239, 480, 1088, True, STREAM, LD256, LD256), (9, 64, 64, True, STREAM, LD256, LD256), (128, 256, 5632, False, STREAM, None, LD256),
           (700, 736, 2080, False, MIDDLE, LD128, LD128), (256, 2048, 5632, True, MIDDLE, LD128, None), (408, 96, 4160, False, SHARED, LD128, LD128),
           (1300, 96, 5024, True, SHARED, None, None), (1024, 896, 5632, False, LARGE, LD256, LD256), (2091, 736, 1952, True, LARGE, None, None),
           (2217, 1152, 3808, True, (LARGE, STREAM, False), None, None), (1796, 1184, 4416, False, (LARGE, STREAM, True), None, None)]
BACKWARD = [(1110, 96, 928, False, STREAM, LD256, LD256), (13, 64, 12288, True, STREAM, LD256, LD256), (1211, 416, 2112, True, MIDDLE, None, LD128),
            (600, 1056, 5536, False, MIDDLE, LD128, None), (900, 96, 4288, True, SHARED, None, LD128), (2977, 864, 5248, True, LARGE, None, LD256),
            (2300, 2080, 5152, False, LARGE, None, None), (3848, 1504, 4352, True, (LARGE, STREAM, True), None, None)]
GRADIENT = [(700, 768, 2016, False, STREAM, (1 << 23) - 64, (1 << 23) - 64), (11, 12288, 96, True, STREAM, None, LD256), (2061, 480, 96, False, MIDDLE, None, (1 << 24) - 64),
            (2048, 2048, 544, True, MIDDLE, None, None), (8192, 2048, 96, True, LARGE, None, LD256), (6000, 2016, 480, False, LARGE, None, None),
            (2478, 1632, 672, True, (MIDDLE, STREAM, False), None, None), (2692, 1536, 608, False, (MIDDLE, STREAM, True), None, None)]


@pytest.mark.parametrize("kept", ["none", "bf16", "e4m3"])
@pytest.mark.parametrize("M,K,F,nk,form,lda,ldw", FORWARD)
def test_forward(M, K, F, nk, form, lda, ldw, kept):
    shape = (F, K) if nk else (K, F)
    lda, ldw = lda or beyond(M, 2, 1 << 23), ldw or beyond(shape[0], 2, 1 << 23)
    assert_form(form, gws.GATED_FWD, M, K, F, nk, kept, (K, shape[1]), (lda, ldw))
    x, wg, wu = some(1, M, K, 1.0), some(2, *shape, 0.02), some(3, *shape, 0.02)
    h, saved = torch.zeros(M, F, dtype=torch.bfloat16, device=DEV), kept_near(kept, M, F)
    gws.gws_gated_fwd(x, wg, wu, h, saved=saved, w_is_nk=nk)
    weights, results = Apart(shape[0], ldw), Apart(M, beyond(M, 2))
    far = results.room(F)
    far_saved, kept_parts = kept_far(kept, saved, results, False)
    gws.gws_gated_fwd(Apart(M, lda).put(x), weights.put(wg), weights.put(wu), far, saved=far_saved, w_is_nk=nk)
    torch.cuda.synchronize()
    assert torch.equal(far, h)
    for a, b in zip(kept_parts, parts(kept, saved)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("kept", ["bf16", "e4m3"])
@pytest.mark.parametrize("M,D,F,nk,form,lda,ldw", BACKWARD)
def test_backward(M, D, F, nk, form, lda, ldw, kept):
    shape = (D, F) if nk else (F, D)
    lda, ldw = lda or beyond(M, 2, 1 << 23), ldw or beyond(shape[0], 2, 1 << 23)
    assert_form(form, gws.GATED_BWD, M, D, F, nk, kept, (D, shape[1]), (lda, ldw))
    dy, w = some(1, M, D, 1e-3), some(2, *shape, 0.02)
    saved = kept_near(kept, M, F, [some(3, M, F, 1.0), some(4, M, F, 1.0)])
    near = [torch.zeros(M, F, dtype=torch.bfloat16, device=DEV) for _ in range(3)]
    gws.gws_gated_bwd(dy, w, saved, near[0], near[1], h=near[2], w_is_nk=nk)
    results = Apart(M, beyond(M, 2))
    far = [results.room(F) for _ in range(3)]
    far_saved, _ = kept_far(kept, saved, results, True)
    gws.gws_gated_bwd(Apart(M, lda).put(dy), Apart(shape[0], ldw).put(w), far_saved, far[0], far[1], h=far[2], w_is_nk=nk)
    torch.cuda.synchronize()
    for a, b in zip(far, near):
        assert torch.equal(a, b)


@pytest.mark.parametrize("M,K,F,nk,form,lda,ldw", GRADIENT)
def test_input_gradient(M, K, F, nk, form, lda, ldw):
    shape = (F, K) if nk else (K, F)
    lda, ldw = lda or beyond(M, 2, 1 << 23), ldw or beyond(shape[0], 2, 1 << 23)
    together = 2 * F + (-F % 64) * 2
    assert_form(form, gws.GATED_BWD_X, M, K, F, nk, "none", (together, shape[1]), (lda, ldw))
    tokens, weights = Apart(M, together), [some(3, *shape, 0.02), some(4, *shape, 0.02)]
    dg, du = (tokens.put(some(s, M, F, 1e-3)) for s in (1, 2))
    dx = torch.zeros(M, K, dtype=torch.bfloat16, device=DEV)
    gws.gws_gated_bwd_x(dg, du, *weights, dx, w_is_nk=nk)
    far_tokens, far_weights, far = Apart(M, lda), Apart(shape[0], ldw), Apart(M, beyond(M, 2)).room(K)
    gws.gws_gated_bwd_x(far_tokens.put(dg), far_tokens.put(du), far_weights.put(weights[0]), far_weights.put(weights[1]), far, w_is_nk=nk)
    torch.cuda.synchronize()
    assert torch.equal(far, dx)
