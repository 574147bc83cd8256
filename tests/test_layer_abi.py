"""Refusals of the norms, the dense layer and the AdamW step: status codes of the C ABI and errors of the binding.  No GPU work is issued here."""
import ctypes
import os

import pytest
import torch

import paper_2505_11170_amd as gws
from paper_2505_11170_amd import binding
from paper_2505_11170_amd.binding import _CAct8, _CGatedSaved, _CAdamWSettings, _CAdamWTensor, _CEpilogue

OK, NULL, SHAPE, ALIGN, FORMAT, LAUNCH, ALIAS = range(7)
INF, NAN = float("inf"), float("nan")


def at(n):
    return 0x10000000 + n * 0x100000   # never dereferenced


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.library_path()):
        from paper_2505_11170_amd.build import build_library
        build_library()
    return binding.load_library()


def test_norm_forward(lib):
    def fwd(x=at(0), M=8, C=100, ldx=104, kind=0, gamma=at(1), beta=at(2), eps=1e-5, y=at(3), ldy=104, mean=at(4), rstd=at(5)):
        return lib.gws_norm_fwd(x, M, C, ldx, kind, gamma, beta, eps, y, ldy, mean, rstd, None)

    assert fwd(M=0) == OK and fwd(M=0, x=None, y=None) == OK
    assert fwd(C=0) == SHAPE and fwd(M=-1) == SHAPE and fwd(C=2 ** 31) == SHAPE and fwd(M=2 ** 31) == SHAPE
    assert fwd(ldx=96) == SHAPE and fwd(ldx=101) == SHAPE and fwd(ldy=100) == SHAPE
    assert fwd(kind=2) == FORMAT and fwd(kind=-1) == FORMAT
    for eps in (0.0, -1e-5, NAN, INF, 1e-60):
        assert fwd(eps=eps) == FORMAT
    assert fwd(x=None) == NULL and fwd(y=None) == NULL and fwd(mean=None) == NULL and fwd(rstd=None) == NULL and fwd(kind=1) == NULL
    assert fwd(x=at(0) + 8) == ALIGN and fwd(y=at(3) + 2) == ALIGN and fwd(gamma=at(1) + 2) == ALIGN and fwd(rstd=at(5) + 1) == ALIGN
    assert fwd(y=at(0), ldy=112) == ALIAS and fwd(y=at(0) + 16) == ALIAS and fwd(mean=at(0)) == ALIAS and fwd(mean=at(5)) == ALIAS
    assert fwd(rstd=at(3)) == ALIAS and fwd(gamma=at(3)) == ALIAS and fwd(beta=at(4)) == ALIAS and fwd(y=at(0), rstd=at(0) + 64) == ALIAS


def test_norm_backward(lib):
    def bwd(dy=at(0), lddy=104, x=at(1), M=8, C=100, ldx=104, kind=0, gamma=at(2), mean=at(3), rstd=at(4), r=at(5), ldr=104, dx=at(6), lddx=104,
            dgamma=at(7), dbeta=at(8), ws=at(9), nbytes=1 << 20):
        return lib.gws_norm_bwd(dy, lddy, x, M, C, ldx, kind, gamma, mean, rstd, r, ldr, dx, lddx, dgamma, dbeta, ws, nbytes, None)

    need = lib.gws_norm_bwd_workspace_bytes(8, 100)
    assert need >= 800 and lib.gws_norm_bwd_workspace_bytes(0, 100) == 0 and lib.gws_norm_bwd_workspace_bytes(8, -1) == 0
    assert bwd(M=-1) == SHAPE and bwd(C=0) == SHAPE and bwd(kind=3) == FORMAT
    for ld in ("lddy", "ldx", "ldr", "lddx"):
        assert bwd(**{ld: 96}) == SHAPE and bwd(**{ld: 108}) == SHAPE
    for p in ("dy", "x", "mean", "rstd", "dx", "ws"):
        assert bwd(**{p: None}) == NULL, p
    assert bwd(nbytes=need - 1) == SHAPE and bwd(ws=at(9) + 8) == ALIGN
    for p in ("dy", "x", "r", "dx"):
        assert bwd(**{p: at(20) + 8}) == ALIGN
    for p in ("gamma", "mean", "rstd", "dgamma", "dbeta"):
        assert bwd(**{p: at(20) + 2}) == ALIGN
    assert bwd(dgamma=at(8)) == ALIAS and bwd(dgamma=at(2)) == ALIAS and bwd(ws=at(0)) == ALIAS and bwd(ws=at(7)) == ALIAS and bwd(ws=at(6)) == ALIAS
    assert bwd(dx=at(1) + 16) == ALIAS and bwd(dx=at(0), lddx=112) == ALIAS and bwd(dx=at(2)) == ALIAS and bwd(dx=at(7)) == ALIAS and bwd(dbeta=at(5)) == ALIAS
    # rows of 50 BF16 columns 100 elements apart look like one row of 50 fp32 ones: still not "the same place"
    assert bwd(C=50, ldx=104, dx=at(2), lddx=56, dgamma=None, dbeta=None) == ALIAS and bwd(M=1, C=96, gamma=at(6), lddx=192) == ALIAS
    # rows that are read again need room for their sums
    assert bwd(C=16392, lddy=16392, ldx=16392, ldr=16392, lddx=16392, dgamma=None, dbeta=None, ws=None) == NULL


def test_dense_forward(lib):
    def fwd(x=at(0), M=8, K=64, ldx=64, w=at(1), N=96, ldw=96, nk=0, y=at(2), ldy=96, bias=at(3), act=1, r=at(4), ldr=96, z=at(5), ldz=96):
        e = _CEpilogue(bias, act, r, ldr, z, ldz)
        return lib.gws_dense_fwd(x, M, K, ldx, w, N, ldw, nk, y, ldy, ctypes.byref(e), None)

    assert fwd(M=0) == OK and fwd(N=0) == OK and fwd(M=0, x=None) == OK
    assert lib.gws_dense_fwd(at(0), 8, 64, 64, at(1), 96, 96, 0, at(2), 96, None, None) == NULL
    assert fwd(act=3) == FORMAT and fwd(act=-1) == FORMAT
    assert fwd(K=0) == SHAPE and fwd(K=48) == SHAPE and fwd(N=80, ldy=80) == SHAPE and fwd(M=2 ** 31) == SHAPE and fwd(M=-2) == SHAPE
    assert fwd(ldx=56) == SHAPE and fwd(ldw=64) == SHAPE and fwd(nk=1, ldw=56) == SHAPE and fwd(ldy=64) == SHAPE and fwd(ldr=98) == SHAPE and fwd(ldz=64) == SHAPE
    for p in ("x", "w", "y"):
        assert fwd(**{p: None}) == NULL
    for p in ("x", "w", "y", "r", "z"):
        assert fwd(**{p: at(20) + 8}) == ALIGN
    assert fwd(bias=at(3) + 2) == ALIGN
    assert fwd(y=at(0)) == ALIAS and fwd(y=at(1)) == ALIAS and fwd(y=at(4), ldy=104) == ALIAS and fwd(y=at(4) + 16) == ALIAS and fwd(z=at(2)) == ALIAS
    assert fwd(z=at(4)) == ALIAS and fwd(z=at(0)) == ALIAS and fwd(bias=at(2)) == ALIAS and fwd(y=at(4), z=at(4)) == ALIAS


def test_dense_backward(lib):
    need = lib.gws_dense_bwd_workspace_bytes(40, 96)
    assert need > 0 and lib.gws_dense_bwd_workspace_bytes(1, 96) == 0 and lib.gws_dense_bwd_workspace_bytes(-1, 96) == 0

    def bwd(dy=at(0), M=40, D=64, lddy=64, wd=at(1), F=96, ldw=64, nk=0, act=1, z=at(2), ldz=96, dz=at(3), lddz=96, h=at(4), ldh=96, db=at(5), ws=at(6), nbytes=need):
        return lib.gws_dense_bwd(dy, M, D, lddy, wd, F, ldw, nk, act, z, ldz, dz, lddz, h, ldh, db, ws, nbytes, None)

    def bwd_h(dy=at(0), M=40, F=96, lddy=96, act=1, z=at(2), ldz=96, dz=at(3), lddz=96, h=at(4), ldh=96, db=at(5), ws=at(6), nbytes=need):
        return lib.gws_dense_bwd_h(dy, M, F, lddy, act, z, ldz, dz, lddz, h, ldh, db, ws, nbytes, None)

    for f in (bwd, bwd_h):
        assert f(M=0, db=None) == OK and f(F=0) == OK and f(M=0, db=at(5) + 1) == ALIGN
        assert f(act=7) == FORMAT and f(M=-1) == SHAPE and f(F=33) == SHAPE and f(lddy=56) == SHAPE and f(ldz=64) == SHAPE and f(lddz=100) == SHAPE and f(ldh=64) == SHAPE
        assert f(dy=None) == NULL and f(z=None) == NULL and f(dz=None) == NULL and f(ws=None) == NULL and f(z=None, act=2) == NULL
        assert f(nbytes=need - 1) == SHAPE and f(ws=at(6) + 4) == ALIGN and f(db=at(5) + 2) == ALIGN
        for p in ("dy", "z", "dz", "h"):
            assert f(**{p: at(20) + 8}) == ALIGN
        assert f(dz=at(4)) == ALIAS and f(dz=at(2) + 16) == ALIAS and f(h=at(2), ldh=104) == ALIAS and f(db=at(2)) == ALIAS and f(db=at(3)) == ALIAS
        assert f(ws=at(3)) == ALIAS and f(ws=at(0)) == ALIAS and f(db=at(6)) == ALIAS and f(dz=at(2), h=at(2)) == ALIAS
    assert bwd(D=0) == SHAPE and bwd(D=40) == SHAPE and bwd(ldw=56) == SHAPE and bwd(nk=1) == SHAPE and bwd(wd=None) == NULL and bwd(wd=at(1) + 2) == ALIGN
    assert bwd(dz=at(0)) == ALIAS and bwd(h=at(1)) == ALIAS and bwd(ws=at(1)) == ALIAS and bwd_h(dz=at(0) + 16) == ALIAS
    assert bwd(act=2, z=None, h=None, dz=None) == NULL


def test_queries_of_the_dense_layers_kernel(lib):
    # host function; without a device for 256 compute units
    form = gws.gws_dense_form
    assert form(gws.DENSE_FWD, 0, 64, 64) == 0 and form(gws.DENSE_FWD, 8, 48, 64) == 0 and form(2, 8, 64, 64) == 0 and form(gws.DENSE_FWD, 8, 64, 64, ldx=56) == 0
    assert form(gws.DENSE_BWD, 8, 64, 96, ldw=56) == 0 and form(gws.DENSE_BWD, 8, 64, 96, True, ldw=88) == 0
    assert form(gws.DENSE_FWD, 8, 32, 64) == gws.GEMM_ANY_SHAPE and form(gws.DENSE_FWD, 8, 64, 64, ldx=1 << 25) == gws.GEMM_ANY_SHAPE
    # the plain product's, or two workgroups a compute unit where that measured faster
    for op in (gws.DENSE_FWD, gws.DENSE_BWD):
        nk = op == gws.DENSE_FWD
        assert form(op, 1, 2048, 5632, nk) == gws.GEMM_STREAM and form(op, 8192, 2048, 5632, nk) == gws.GEMM_LARGE and form(op, 514, 64, 3392, not nk) == gws.GEMM_MIDDLE
    assert [form(gws.DENSE_FWD, m, k, n, nk) for m, k, n, nk in ((798, 672, 5632, True), (1118, 352, 4864, False), (5469, 5632, 800, False), (7474, 2304, 1504, False))] == \
        [gws.DENSE_SHARED] * 3 + [gws.GEMM_NARROW]
    assert [form(gws.DENSE_BWD, m, k, n, True) for m, k, n in ((5299, 896, 1536), (2381, 288, 2528), (3281, 5632, 4320))] == [gws.DENSE_SHARED] * 2 + [gws.GEMM_LARGE_EDGE]


def tensor(**over):
    c = _CAdamWTensor(p=at(0), w=at(1), g=at(2), g_is_fp32=0, m=at(3), v=at(4), rows=10, cols=70, ld=72, lr_scale=1.0, weight_decay=0.1, seed=1)
    for k, v in over.items():
        setattr(c, k, v)
    return c


def in8(**over):
    return tensor(**{**dict(m=None, v=None, m8=_CAct8(at(5), at(6), 72, 3), v8=_CAct8(at(7), at(8), 72, 3)), **over})


def test_adamw(lib):
    def step(t=None, n=1, lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, step=1, scale=None):
        s = _CAdamWSettings(lr, beta1, beta2, eps, step, scale)
        return lib.gws_adamw((_CAdamWTensor * 1)(tensor() if t is None else t), n, ctypes.byref(s), None)

    assert step(n=0) == OK and step(n=-1) == SHAPE and step(tensor(rows=0)) == OK and step(tensor(cols=0, p=None)) == OK
    assert lib.gws_adamw(None, 1, ctypes.byref(_CAdamWSettings(1e-3, 0.9, 0.99, 1e-8, 1, None)), None) == NULL
    assert lib.gws_adamw((_CAdamWTensor * 1)(tensor()), 1, None, None) == NULL
    for bad in (dict(lr=NAN), dict(lr=INF), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=NAN), dict(eps=0.0), dict(eps=-1.0), dict(eps=NAN), dict(eps=1e-60), dict(step=0)):
        assert step(**bad) == FORMAT, bad
    assert step(tensor(lr_scale=INF)) == FORMAT and step(tensor(weight_decay=NAN)) == FORMAT
    assert step(scale=at(9) + 2) == ALIGN and step(scale=at(0) + 8) == ALIAS
    for make in (tensor, in8):
        assert step(make(rows=-1)) == SHAPE and step(make(cols=2 ** 31)) == SHAPE and step(make(ld=64)) == SHAPE and step(make(ld=71)) == SHAPE
        assert step(make(rows=2 ** 30, cols=2 ** 30, ld=2 ** 30)) == SHAPE
        assert step(make(p=None)) == NULL and step(make(g=None)) == NULL
        for p in ("p", "w", "g"):
            assert step(make(**{p: at(20) + 8})) == ALIGN
        assert step(make(w=at(0))) == ALIAS and step(make(g=at(0))) == ALIAS and step(make(g=at(1))) == ALIAS
    assert step(tensor(m=None)) == NULL and step(tensor(v=None)) == NULL and step(tensor(m=at(3) + 4)) == ALIGN and step(tensor(m=at(4))) == ALIAS and step(tensor(v=at(2))) == ALIAS
    assert step(in8(m=at(3))) == FORMAT and step(tensor(m8=_CAct8(at(5), at(6), 72, 3))) == FORMAT
    assert step(in8(v8=_CAct8(None, at(8), 72, 3))) == NULL and step(in8(v8=_CAct8(at(7), None, 72, 3))) == NULL
    assert step(in8(m8=_CAct8(at(5), at(6), 80, 3))) == SHAPE and step(in8(m8=_CAct8(at(5), at(6), 72, 2))) == SHAPE and step(in8(m8=_CAct8(at(5), at(6), 72, 4))) == SHAPE
    assert step(in8(m8=_CAct8(at(5) + 4, at(6), 72, 3))) == ALIGN and step(in8(m8=_CAct8(at(7), at(6), 72, 3))) == ALIAS and step(in8(v8=_CAct8(at(7), at(6), 72, 3))) == ALIAS
    # sizes of more workgroups than a launch has
    assert step(tensor(rows=2 ** 30, cols=40, ld=40)) == SHAPE and step(in8(rows=2 ** 30, cols=8, ld=8, m8=_CAct8(at(5), at(6), 8, 1), v8=_CAct8(at(7), at(8), 8, 1))) == SHAPE


def test_adamw_refuses_a_tensor_that_it_was_given_before(lib):
    s = ctypes.byref(_CAdamWSettings(1e-3, 0.9, 0.99, 1e-8, 1, None))

    def step(*t):
        return lib.gws_adamw((_CAdamWTensor * len(t))(*t), len(t), s, None)

    far = lambda buffer, i: buffer * 2 ** 32 + 2 ** 16 * i  # noqa: E731 - 900 tensors of one buffer stay below the next one's
    good = lambda i: tensor(p=far(1, i), w=far(2, i), m=far(3, i), v=far(4, i))  # noqa: E731
    for n in (1, 7, 900):
        before = [good(i) for i in range(n)]
        assert step(*before, good(n - 1)) == ALIAS and step(*before, good(0)) == ALIAS
        for field in ("p", "w", "m", "v"):
            t = good(n)
            setattr(t, field, getattr(good(0), field))
            assert step(*before, t) == ALIAS, field
            if field != "w":
                c = in8(p=at(20), w=at(21), m8=_CAct8(far(3, 0), at(6), 72, 3))          # codes where the first one's m lies
                assert step(*before, c) == ALIAS
        assert step(*before, tensor(rows=0, p=far(1, 0)), tensor(ld=64)) == SHAPE       # an empty one may be anything


def test_gradient_norm(lib):
    one = (_CAdamWTensor * 1)(tensor(p=None, m=None, v=None, w=None))
    need = lib.gws_grad_norm_workspace_bytes(one, 1)
    assert need > 0 and need % 16 == 0 and lib.gws_grad_norm_workspace_bytes(one, 0) == 0 and lib.gws_grad_norm_workspace_bytes(None, 1) == 0

    def norm(t=one, n=1, limit=1.0, out=at(10), ws=at(11), nbytes=need):
        return lib.gws_grad_norm(t, n, limit, out, ws, nbytes, None)

    assert norm(n=-1) == SHAPE and norm(t=None) == NULL and norm(out=None) == NULL and norm(ws=None) == NULL
    assert norm(out=at(10) + 2) == ALIGN and norm(ws=at(11) + 8) == ALIGN and norm(nbytes=need - 1) == SHAPE
    assert norm(limit=NAN) == FORMAT and norm(limit=INF) == FORMAT
    assert norm(out=at(11)) == ALIAS and norm(out=at(2)) == ALIAS and norm(ws=at(2)) == ALIAS
    assert norm((_CAdamWTensor * 1)(tensor(g=None))) == NULL and norm((_CAdamWTensor * 1)(tensor(g=at(2) + 4))) == ALIGN and norm((_CAdamWTensor * 1)(tensor(ld=64))) == SHAPE


def test_binding_refuses_what_the_kernels_would_misread(lib):
    b = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    f = lambda *s: torch.zeros(*s)  # noqa: E731
    x, v = b(4, 64), f(64)
    for bad in (dict(y=b(4, 72)), dict(y=f(4, 64)), dict(y=b(64, 4).t()), dict(gamma=f(63)), dict(gamma=b(64)), dict(beta=f(128)[::2]), dict(rstd=f(5), mean=f(4))):
        with pytest.raises(ValueError):
            gws.gws_norm_fwd(x, **{**dict(y=b(4, 64), gamma=v, beta=v, mean=f(4), rstd=f(4)), **bad})
    for bad in (dict(residual=b(4, 32)), dict(dgamma=f(4)), dict(dx=f(4, 64)), dict(dy=b(3, 64)), dict(workspace=f(64)[::2])):
        with pytest.raises(ValueError):
            gws.gws_norm_bwd(**{**dict(dy=x, x=x, dx=b(4, 64), rstd=f(4), mean=f(4), dgamma=v, workspace=f(4096)), **bad})
    for bad in (dict(w=b(32, 64)), dict(y=b(4, 32)), dict(bias=f(32)), dict(bias=b(96)), dict(residual=b(4, 64)), dict(z=f(4, 96)), dict(w=b(96, 64))):
        with pytest.raises(ValueError):
            gws.gws_dense_fwd(x, **{**dict(w=b(64, 96), y=b(4, 96), bias=f(96)), **bad})
    for bad in (dict(wd=b(64, 96)), dict(z=b(4, 64)), dict(dz=b(5, 96)), dict(h=f(4, 96)), dict(dbias=b(96))):
        with pytest.raises(ValueError):
            gws.gws_dense_bwd(x, **{**dict(wd=b(96, 64), z=b(4, 96), dz=b(4, 96), act=gws.ACT_SILU), **bad})
    # host memory, which a kernel cannot read
    with pytest.raises(ValueError, match="device"):
        gws.gws_norm_fwd(x, b(4, 64))
    with pytest.raises(ValueError, match="device"):
        gws.gws_dense_bwd_h(x, None, None, dbias=v)
    a8 = lambda: gws.Act8(torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(4, 2, dtype=torch.uint8))  # noqa: E731
    good = dict(p=f(4, 64), g=b(4, 64), m=f(4, 64), v=f(4, 64))
    for bad in (dict(g=b(4, 72)[:, :64]), dict(m=f(4, 72)), dict(m=a8()), dict(p=b(4, 64)), dict(w=f(4, 64)), dict(g=torch.zeros(4, 64, dtype=torch.float16)), dict(v=f(64, 4).t()),
                dict(m=a8(), v=gws.Act8(torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(4, 1, dtype=torch.uint8))), dict(p=f(2, 2, 64))):
        with pytest.raises(ValueError):
            gws.pack_adamw([gws.AdamWTensor(**{**good, **bad})])
    packed = gws.pack_adamw([gws.AdamWTensor(**good), gws.AdamWTensor(p=f(3), g=f(3), m=f(3), v=f(3))])
    assert len(packed) == 2 and (packed.arr[1].rows, packed.arr[1].cols, packed.arr[1].ld, packed.arr[1].g_is_fp32) == (1, 3, 8, 1)
    with pytest.raises(ValueError):
        gws.gws_adamw(packed, 1e-3, 1, grad_scale=torch.zeros(2))
    with pytest.raises(ValueError, match="device"):
        gws.gws_adamw(packed, 1e-3, 1)


def test_a_gate_s_gradients_do_not_lie_on_codes(lib):
    """Not even where the codes' rows lie as far apart as theirs: at the same place only a matrix of the same rows and bytes is."""
    saved = _CGatedSaved(g8=_CAct8(at(5), at(6), 128, 2), u8=_CAct8(at(7), at(8), 128, 2))
    for n in (5, 7):
        out = [at(n), at(10)] if n == 5 else [at(10), at(n)]
        assert lib.gws_gated_bwd_h(at(0), 8, 64, 64, gws.ACT_SILU, ctypes.byref(saved), *out, 64, None, 0, None) == ALIAS
        assert lib.gws_gated_bwd(at(0), 8, 64, 64, at(1), 64, 64, 0, gws.ACT_SILU, ctypes.byref(saved), *out, 64, None, 0, None) == ALIAS


def test_adamw_refuses_scales_that_it_was_given_before(lib):
    """Block scales are written too: of m or v, of a tensor before or of what another one has at the same address."""
    s = ctypes.byref(_CAdamWSettings(1e-3, 0.9, 0.99, 1e-8, 1, None))

    def step(*t):
        return lib.gws_adamw((_CAdamWTensor * len(t))(*t), len(t), s, None)

    far = lambda buffer, i: buffer * 2 ** 32 + 2 ** 16 * i  # noqa: E731
    good = lambda i, m=None, v=None: in8(p=far(1, i), w=far(2, i), m8=_CAct8(far(3, i), m or far(4, i), 72, 3), v8=_CAct8(far(5, i), v or far(6, i), 72, 3))  # noqa: E731
    for n in (1, 7, 400):
        before = [good(i) for i in range(n)]
        for i in (0, n - 1):
            for taken in (far(4, i), far(6, i), far(3, i), far(5, i), far(1, i)):
                assert step(*before, good(n, m=taken)) == ALIAS and step(*before, good(n, v=taken)) == ALIAS
            for field in ("p", "m", "v"):
                t = tensor(p=far(7, 0), w=far(8, 0), m=far(9, 0), v=far(10, 0))
                setattr(t, field, far(4, i))
                assert step(*before, t) == ALIAS, field
        assert step(*before, good(n), tensor(ld=64)) == SHAPE       # apart: only the one behind is refused
