"""What the entry points of the gated block and of 8-bit activations refuse, and that nothing is launched then (no GPU work is issued here);
and the definition of the 8-bit form against plain arithmetic."""
import ctypes
import math

import pytest
import torch

import gated_ref as ref
from gpu_util import ensure_built
from paper_2505_11170_amd import binding
from paper_2505_11170_amd.binding import Act8, GatedSaved, _CAct8, _CGatedSaved, _CTensor

OK, NULL, SHAPE, ALIGN, FORMAT, LAUNCH, ALIAS = range(7)
MB = 1 << 20


@pytest.fixture(scope="module")
def lib():
    ensure_built()
    return binding.load_library()


def at(n):
    return 0x10000000 + n * MB     # never dereferenced: every call below is refused first, or has nothing to do


def act8(codes=at(20), xscale=at(21), ldc=64, lds=2):
    return _CAct8(codes, xscale, ldc, lds)


def bf16(g=at(30), u=at(31), ldg=64, ldu=64):
    return _CGatedSaved(g, u, ldg, ldu, _CAct8(), _CAct8())


def in8(g8=None, u8=None, g=None, u=None):
    return _CGatedSaved(g, u, 64, 64, g8 or act8(), u8 or act8(at(22), at(23)))


def test_act8(lib):
    def enc(x=at(0), M=8, C=64, ldx=64, **o):
        return lib.gws_act8_encode(x, M, C, ldx, ctypes.byref(act8(**o)), None)

    def dec(x=at(0), M=8, C=64, ldx=64, **o):
        return lib.gws_act8_decode(ctypes.byref(act8(**o)), M, C, x, ldx, None)

    for f in (enc, dec):
        assert f(M=0) == OK and f(C=0) == OK
        assert f(M=-1) == SHAPE and f(C=2 ** 31) == SHAPE and f(ldx=60) == SHAPE and f(ldx=56) == SHAPE
        assert f(ldc=56) == SHAPE and f(ldc=65) == SHAPE and f(lds=1) == SHAPE and f(C=65, ldx=72, ldc=72) == SHAPE
        assert f(x=None) == NULL and f(codes=None) == NULL and f(xscale=None) == NULL
        assert f(x=at(0) + 8) == ALIGN and f(codes=at(20) + 4) == ALIGN
        assert f(codes=at(0)) == ALIAS and f(xscale=at(0) + 100) == ALIAS
    assert enc(xscale=at(20) + 3) == ALIAS
    assert lib.gws_act8_encode(at(0), 8, 64, 64, None, None) == NULL and lib.gws_act8_decode(None, 8, 64, at(0), 64, None) == NULL


def test_forward(lib):
    def fwd(x=at(0), M=8, K=64, ldx=64, wg=at(1), wu=at(2), F=64, ldw=64, nk=0, act=0, h=at(3), ldh=64, saved=None):
        return lib.gws_gated_fwd(x, M, K, ldx, wg, wu, F, ldw, nk, act, h, ldh, None if saved is None else ctypes.byref(saved), None)

    assert fwd(M=0) == OK and fwd(F=0) == OK and fwd(M=0, x=None) == OK
    assert fwd(act=2) == FORMAT and fwd(act=-1) == FORMAT
    assert fwd(M=-1) == SHAPE and fwd(K=0) == SHAPE and fwd(K=48) == SHAPE and fwd(F=48) == SHAPE and fwd(M=2 ** 31) == SHAPE
    assert fwd(ldx=56) == SHAPE and fwd(ldx=66) == SHAPE and fwd(ldw=32) == SHAPE and fwd(ldh=32) == SHAPE and fwd(K=96, ldx=96, nk=1) == SHAPE
    for n in ("x", "wg", "wu", "h"):
        assert fwd(**{n: None}) == NULL and fwd(**{n: at(9) + 8}) == ALIGN
    assert fwd(h=at(0)) == ALIAS and fwd(h=at(1) + 16) == ALIAS and fwd(h=at(2)) == ALIAS
    assert fwd(saved=bf16(u=None)) == NULL and fwd(saved=in8(g8=act8(xscale=None))) == NULL and fwd(saved=_CGatedSaved()) == NULL
    assert fwd(saved=in8(g=at(30), u=at(31))) == FORMAT                                      # both forms at once
    assert fwd(saved=bf16(ldg=56)) == SHAPE and fwd(saved=in8(u8=act8(at(22), at(23), 64, 1))) == SHAPE
    assert fwd(saved=bf16(g=at(30) + 2)) == ALIGN and fwd(saved=in8(g8=act8(codes=at(20) + 2))) == ALIGN
    assert fwd(saved=bf16(g=at(3))) == ALIAS and fwd(saved=bf16(g=at(31))) == ALIAS and fwd(saved=bf16(u=at(0))) == ALIAS
    assert fwd(saved=in8(u8=act8())) == ALIAS and fwd(saved=in8(g8=act8(xscale=at(3)))) == ALIAS
    # rows that lie between each other's
    assert fwd(ldh=128, saved=bf16(g=at(3) + 64, ldg=128)) == ALIAS and fwd(ldh=128, saved=bf16(g=at(3) + 144, ldg=128)) == ALIAS


def test_backward(lib):
    def bwd(dy=at(0), M=8, D=64, lddy=64, wd=at(1), F=64, ldw=64, nk=0, act=0, saved=None, dg=at(3), du=at(4), ldd=64, h=at(5), ldh=64):
        return lib.gws_gated_bwd(dy, M, D, lddy, wd, F, ldw, nk, act, ctypes.byref(saved or bf16()), dg, du, ldd, h, ldh, None)

    def bwd_h(dy=at(0), M=8, F=64, lddy=64, act=0, saved=None, dg=at(3), du=at(4), ldd=64, h=at(5), ldh=64):
        return lib.gws_gated_bwd_h(dy, M, F, lddy, act, ctypes.byref(saved or bf16()), dg, du, ldd, h, ldh, None)

    for f in (bwd, bwd_h):
        assert f(M=0) == OK and f(F=0) == OK and f(act=7) == FORMAT
        assert f(M=-1) == SHAPE and f(F=33) == SHAPE and f(lddy=32) == SHAPE and f(ldd=32) == SHAPE and f(ldd=68) == SHAPE and f(ldh=32) == SHAPE
        assert f(h=None, ldh=0, dg=None) == NULL and f(du=None) == NULL and f(dy=None) == NULL and f(saved=bf16(g=None)) == NULL
        for n in ("dy", "dg", "du", "h"):
            assert f(**{n: at(9) + 8}) == ALIGN
        assert f(dg=at(4)) == ALIAS and f(h=at(3)) == ALIAS and f(saved=bf16(ldg=72), dg=at(30)) == ALIAS and f(dg=at(30) + 16) == ALIAS
        assert f(saved=in8(), du=at(20)) == ALIAS and f(saved=in8(), h=at(23)) == ALIAS
    assert lib.gws_gated_bwd(at(0), 8, 64, 64, at(1), 64, 64, 0, 0, None, at(3), at(4), 64, None, 0, None) == NULL
    assert bwd(D=0) == SHAPE and bwd(D=40) == SHAPE and bwd(ldw=32) == SHAPE and bwd(F=96, ldd=96, ldh=96, nk=1) == SHAPE
    assert bwd(wd=None) == NULL and bwd(wd=at(1) + 4) == ALIGN
    assert bwd(dg=at(0)) == ALIAS and bwd(h=at(1)) == ALIAS and bwd_h(dg=at(0) + 16) == ALIAS


def test_input_gradient(lib):
    def dx(dg=at(0), du=at(1), M=8, F=64, ldd=64, wg=at(2), wu=at(3), K=64, ldw=64, nk=0, dx=at(4), ldx=64):
        return lib.gws_gated_bwd_x(dg, du, M, F, ldd, wg, wu, K, ldw, nk, dx, ldx, None)

    assert dx(M=0) == OK and dx(K=0) == OK
    assert dx(F=0) == SHAPE and dx(F=48) == SHAPE and dx(K=16) == SHAPE and dx(M=-4) == SHAPE
    assert dx(ldd=32) == SHAPE and dx(ldw=32) == SHAPE and dx(ldx=62) == SHAPE and dx(K=96, ldx=96, nk=1) == SHAPE
    for n in ("dg", "du", "wg", "wu", "dx"):
        assert dx(**{n: None}) == NULL and dx(**{n: at(9) + 2}) == ALIGN
    for n in range(4):
        assert dx(dx=at(n)) == ALIAS


def test_weight_gradient(lib):
    base = dict(dw=at(40), rows=256, cols=512, ld=512, seed=1)

    def desc(**over):
        c = _CTensor()
        for k, v in {**base, **over}.items():
            setattr(c, k, v)
        return ctypes.byref(c)

    def call(a=None, dy=at(50), M=128, ldy=512, w=None, nk=0, ws=at(60), n=128 * 256 * 2):
        return lib.gws_linear_bwd_w_act8(ctypes.byref(a or act8(ldc=256, lds=8)), dy, M, ldy, w or desc(), nk, 0, ws, n, None)

    assert lib.gws_linear_bwd_w_act8_workspace_bytes(desc(), 0, 128) >= 128 * 256 * 2
    assert lib.gws_linear_bwd_w_act8_workspace_bytes(desc(), 1, 128) >= 128 * 512 * 2
    assert lib.gws_linear_bwd_w_act8_workspace_bytes(None, 0, 128) == 0 and lib.gws_linear_bwd_w_act8_workspace_bytes(desc(), 0, 100) == 0
    assert call(M=0) == SHAPE and call(M=100) == SHAPE and call(ldy=256) == SHAPE and call(w=desc(rows=128)) == SHAPE
    assert call(n=128 * 256 * 2 - 1) == SHAPE and call(a=act8(ldc=128, lds=8)) == SHAPE and call(a=act8(ldc=256, lds=7)) == SHAPE
    assert call(dy=None) == NULL and call(ws=None) == NULL and call(a=act8(codes=None)) == NULL and call(w=desc(dw=None)) == NULL
    assert call(w=desc(dbt=at(70))) == NULL and call(ws=at(60) + 16) == ALIGN and call(a=act8(codes=at(20) + 4, ldc=256, lds=8)) == ALIGN
    assert call(ws=at(50)) == ALIAS and call(ws=at(40)) == ALIAS and call(ws=at(20)) == ALIAS and call(ws=at(21)) == ALIAS
    assert call(w=desc(dw=at(20))) == ALIAS and call(w=desc(dbt=at(60), scale=at(71))) == ALIAS
    assert lib.gws_linear_bwd_w_act8(None, at(50), 128, 512, desc(), 0, 0, at(60), MB, None) == NULL


def test_workspace_of_sizes_that_the_weight_gradient_refuses(lib):
    def desc(rows, cols):
        return ctypes.byref(_CTensor(dw=at(40), rows=rows, cols=cols, ld=cols, seed=1))

    assert lib.gws_linear_bwd_w_act8_workspace_bytes(desc(256, 512), 0, 2 ** 31 - 64) >= (2 ** 31 - 64) * 256 * 2
    for M, rows, cols in ((2 ** 31, 256, 512), (2 ** 40, 256, 512), (64, 2 ** 31, 256), (64, 256, 2 ** 31)):
        a = act8(ldc=rows, lds=rows // 32)
        assert lib.gws_linear_bwd_w_act8(ctypes.byref(a), at(50), M, cols, desc(rows, cols), 0, 0, at(60), MB, None) == SHAPE
        assert lib.gws_linear_bwd_w_act8_workspace_bytes(desc(rows, cols), 0, M) == 0


def test_python_shapes():
    z = lambda *s, d=torch.bfloat16: torch.zeros(*s, dtype=d)  # noqa: E731
    a = Act8(z(4, 64, d=torch.uint8), z(4, 2, d=torch.uint8))
    with pytest.raises(ValueError):
        binding.gws_act8_encode(z(4, 96), a)
    with pytest.raises(ValueError):
        binding.gws_act8_decode(Act8(a.codes, a.codes), z(4, 64))
    with pytest.raises(ValueError):
        binding.gws_gated_fwd(z(4, 64), z(64, 96), z(64, 64), z(4, 96))
    with pytest.raises(ValueError):
        binding.gws_gated_fwd(z(4, 64), z(64, 96), z(64, 192)[:, :96], z(4, 96))                      # leading dimensions differ
    with pytest.raises(ValueError):
        binding.gws_gated_fwd(z(4, 64), z(64, 64), z(64, 64), z(4, 64), saved=GatedSaved(g=z(4, 32), u=z(4, 64)))
    with pytest.raises(ValueError):
        binding.gws_gated_bwd(z(4, 64), z(96, 64), GatedSaved(g8=a, u8=a), z(4, 96), z(4, 96))
    with pytest.raises(ValueError):
        binding.gws_gated_bwd_h(z(4, 64), GatedSaved(g8=a, u8=a), z(4, 64), z(4, 128)[:, :64])
    with pytest.raises(ValueError):
        binding.gws_gated_bwd_x(z(4, 96), z(4, 96), z(64, 96), z(64, 96), z(4, 96))
    with pytest.raises(ValueError):
        binding.gws_linear_bwd_w_act8(a, z(4, 256), binding.TensorDesc(rows=256, cols=256, seed=0), 0, None)


def test_python_shapes_of_the_weight_gradient():
    # columns of a wider buffer have a leading dimension that fits any weight: the shapes have to
    z = lambda *s, d=torch.bfloat16: torch.zeros(*s, dtype=d)  # noqa: E731
    for nk in (False, True):
        rows, cols, K, N = (512, 256, 256, 512) if nk else (256, 512, 256, 512)
        x = Act8(z(128, K, d=torch.uint8), z(128, K // 32, d=torch.uint8))

        def call(dy, dw=None, x=x):
            w = binding.TensorDesc(rows=rows, cols=cols, seed=0, dw=z(rows, cols) if dw is None else dw)
            binding.gws_linear_bwd_w_act8(x, dy, w, 0, z(1 << 20, d=torch.uint8), w_is_nk=nk)

        for dy in (z(128, 1024)[:, :256], z(128, 1024)[:, :N + 8], z(128, N - 256), z(128, K)):
            with pytest.raises(ValueError, match="do not fit"):
                call(dy)
        for dw in (z(cols, rows), z(rows, 2 * cols)[:, : cols - 32], z(rows - 32, cols)):
            with pytest.raises(ValueError, match="do not fit"):
                call(z(128, N), dw)
        with pytest.raises(ValueError):
            call(z(192, N))                                                                           # other tokens than X's


def test_python_types_and_strides():
    # what the kernels would read as something else: other types, columns apart, each argument of each call in turn
    def call(name, **bad):
        z = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
        b = lambda *s: torch.zeros(*s, dtype=torch.uint8)  # noqa: E731
        t = dict(x=z(4, 64), wg=z(64, 64), wu=z(64, 64), h=z(4, 64), g=z(4, 64), u=z(4, 64), dg=z(4, 64), du=z(4, 64), codes=b(4, 64), xscale=b(4, 2))
        t.update({k: v(t[k]) for k, v in bad.items()})
        a = lambda: Act8(t["codes"], t["xscale"])  # noqa: E731
        {"encode": lambda: binding.gws_act8_encode(t["x"], a()), "decode": lambda: binding.gws_act8_decode(a(), t["x"]),
         "fwd": lambda: binding.gws_gated_fwd(t["x"], t["wg"], t["wu"], t["h"], 9, saved=GatedSaved(g=t["g"], u=t["u"])),
         "bwd": lambda: binding.gws_gated_bwd(t["x"], t["wg"], GatedSaved(g=t["g"], u=t["u"]), t["dg"], t["du"], 9, h=t["h"]),
         "bwd8": lambda: binding.gws_gated_bwd(t["x"], t["wg"], GatedSaved(g8=a(), u8=a()), t["dg"], t["du"], 9),
         "bwd_h": lambda: binding.gws_gated_bwd_h(t["x"], GatedSaved(g=t["g"], u=t["u"]), t["dg"], t["du"], 9, h=t["h"]),
         "bwd_x": lambda: binding.gws_gated_bwd_x(t["dg"], t["du"], t["wg"], t["wu"], t["x"]),
         "bwd_w": lambda: binding.gws_linear_bwd_w_act8(a(), t["x"], binding.TensorDesc(rows=64, cols=64, seed=0), 0, None)}[name]()

    def apart(v):
        return torch.zeros(v.shape[0], 2 * v.shape[1], dtype=v.dtype)[:, ::2]

    takes = {"encode": ("x", "codes", "xscale"), "decode": ("x", "codes", "xscale"), "fwd": ("x", "wg", "wu", "h", "g", "u"),
             "bwd": ("x", "wg", "g", "u", "dg", "du", "h"), "bwd8": ("codes", "xscale"), "bwd_h": ("x", "g", "u", "dg", "du", "h"),
             "bwd_x": ("dg", "du", "wg", "wu", "x"), "bwd_w": ("x", "codes", "xscale")}
    for name, args in takes.items():
        for arg in args:
            for wrong in (apart, lambda v: v.float(), lambda v: v.half()):
                with pytest.raises(ValueError, match="next to each other"):
                    call(name, **{arg: wrong})
    for one_byte in (torch.float8_e4m3fn, torch.int8):
        binding._check_bytes(torch.zeros(4, 64, dtype=torch.uint8).view(one_byte))
    binding._check_plain(torch.zeros(4, 8, dtype=torch.bfloat16)[:, ::8])                           # one column has no next


def test_the_example_refuses_what_its_weight_gradients_do():
    # before any buffer is made, not in the first backward pass
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "gated_ffn.py")
    spec = importlib.util.spec_from_file_location("gated_ffn_sizes", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    ensure_built()
    for tokens, width, block in ((1021, 256, 512), (0, 256, 512), (1024, 320, 512), (1024, 256, 544)):
        with pytest.raises(ValueError, match="multiple of 64 tokens"):
            example.GatedFFN(tokens, width, block)


def test_definition_of_the_8_bit_form():
    # the reference that the GPU tests compare with, against torch's own casts where it has them
    gen = torch.Generator().manual_seed(1)
    v = (torch.randn(400, 96, generator=gen) * torch.exp(6.0 * torch.randn(400, 1, generator=gen))).bfloat16().double()
    codes, xs = ref.encode(v)
    x = ref.pow2(xs.long() - 127)[:, ref.blocks(96)]
    assert torch.equal(codes, (v / x).float().to(torch.float8_e4m3fn).view(torch.uint8))
    assert torch.equal(ref.decode(codes, xs), codes.view(torch.float8_e4m3fn).double() * x)
    assert torch.equal(xs.view(torch.float8_e8m0fnu).double(), ref.pow2(xs.long() - 127))
    # the scale: doubling it is never needed, halving it would overflow (or is below the least)
    top = v.abs().reshape(400, 3, 32).amax(dim=2)
    s = ref.pow2(xs.long() - 127)
    assert (top / s <= 464).all() and ((top / s > 232) | (xs == 10) | (top == 0)).all()
    # values: within half a spacing, and BF16 again without a change
    d = ref.decode(codes, xs)
    assert torch.equal(d.bfloat16().double(), d)
    assert ((d - v).abs() <= torch.maximum(v.abs() * 2.0 ** -4, x * 2.0 ** -10)).all()
    z = torch.tensor([[0.0, -0.0] * 16 + [math.nan] + [1.0] * 31])
    codes, xs = ref.encode(z.double())
    assert xs.tolist() == [[127, 255]] and codes[0, :2].tolist() == [0, 128] and (codes[0, 32:] == 127).all()


def test_gated_kernels_use_no_scratch():
    # a kernel with scratch starts later, and the tiles leave no registers over
    from test_kernel_resources import kernels
    mine = [k for k in kernels().values() if any(p in k[".name"] for p in ("gated", "act8"))]
    assert len(mine) > 80 and not [k[".name"] for k in mine if k[".private_segment_fixed_size"] != 0]


def test_h_is_kept_in_the_caches_for_the_product_that_reads_it():
    # by the time of the call and that product together: past the caches only where H outgrows them
    ensure_built()
    past = binding.gws_gated_past_caches
    for kept in (0, 1, 2):
        for M in (1, 1024, 4096, 8192, 12288, 15360):
            assert not past(binding.GATED_FWD, M, 2048, 5632, True, kept)
        for M in (16384, 32768):
            assert past(binding.GATED_FWD, M, 2048, 5632, True, kept)
    assert not past(binding.GATED_FWD, 16384, 768, 2048) and not past(binding.GATED_BWD_X, 32768, 2048, 5632)
    assert not past(binding.GATED_FWD, 32768, 2048, 5600 + 16)                                      # refused


def test_gradients_are_kept_in_the_caches_where_what_reads_them_waits_for_memory():
    # by the time of the whole backward pass: past the caches where the products are bound by the matrix cores
    ensure_built()
    past = binding.gws_gated_past_caches
    for kept in (1, 2):
        for M, D, F in ((2048, 768, 2048), (4096, 768, 2048), (8192, 768, 2048), (16384, 768, 2048), (4096, 768, 2304)):
            assert not past(binding.GATED_BWD, M, D, F, True, kept)
        for M, D, F in ((2048, 1024, 4096), (8192, 1024, 4096), (1024, 2048, 5632), (4096, 2048, 5632), (8192, 2048, 5632)):
            assert past(binding.GATED_BWD, M, D, F, True, kept)


def test_query_of_the_chosen_kernel():
    # a host function; without a device for 256 compute units
    ensure_built()
    form = binding.gws_gated_form
    assert form(binding.GATED_FWD, 8192, 2048, 5632, True, 2)[0] == binding.GATED_LARGE
    assert form(binding.GATED_FWD, 1021, 768, 2048, False, 1)[0] == binding.GATED_MIDDLE
    assert form(binding.GATED_FWD, 1, 2048, 5632, True) == (binding.GATED_STREAM, 1, 2) or form(binding.GATED_FWD, 1, 2048, 5632, True) == (binding.GATED_STREAM, 1, 4)
    assert form(binding.GATED_FWD, 8192, 32, 5632)[0] == binding.GATED_ANY and form(binding.GATED_FWD, 4, 2048, 64, True, lda=1 << 24)[0] == binding.GATED_ANY
    assert form(binding.GATED_BWD_X, 8192, 2048, 5632, True)[0] == binding.GATED_LARGE
    assert binding.gws_gated_forms(binding.GATED_FWD, 1021, 768, 2048, False, 1) == ((binding.GATED_MIDDLE, 0, 0), 0, False)
    assert binding.gws_gated_forms(binding.GATED_FWD, 2217, 1152, 3808, True) == ((binding.GATED_LARGE, 0, 0), binding.GATED_STREAM, False)
    assert binding.gws_gated_forms(binding.GATED_FWD, 2914, 1376, 3424, True) == ((binding.GATED_LARGE, 0, 0), binding.GATED_SHARED, True)
    for bad in ((3, 4, 64, 64), (0, 0, 64, 64), (0, 4, 48, 64), (1, 4, 64, 64, False, 0), (0, 4, 64, 64, False, 3)):
        assert form(*bad)[0] == 0
    assert form(binding.GATED_FWD, 4, 64, 64, lda=56)[0] == 0
