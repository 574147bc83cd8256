"""The dense layer, forward and backward, against 64 bits (bounds: layer_ref.py)."""
import math

import pytest
import torch

import gated_ref
import layer_ref as ref
import paper_2505_11170_amd as gws
from gated_ref import assert_within
from gpu_util import DEV, ensure_built
from test_gpu_gated import rand, room
from test_gpu_norm import odd_start, vec

pytestmark = pytest.mark.gpu
ACTS = [gws.ACT_NONE, gws.ACT_SILU, gws.ACT_GELU_TANH]


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_built()


def weight(seed, K, N, nk, pad=0, std=None):
    std = std or 1.0 / math.sqrt(K)
    return rand(seed, N, K, std, K + pad) if nk else rand(seed, K, N, std, N + pad)


def check_fwd(M, K, N, nk, act, bias=True, residual=True, keep=True, pad=0, in_place=False, check=True):
    x, w = rand(1, M, K, 1.0, K + pad), weight(2, K, N, nk, pad)
    b = odd_start(vec(3, N)) if bias else None
    r = rand(4, M, N, 1.0, N + 2 * pad) if residual else None
    y, whole = (r.clone(), None) if in_place else room(M, N, N + pad)
    z, zwhole = room(M, N, N + 3 * pad) if keep else (None, None)
    if in_place:
        r = y
        r0 = r.clone()
    gws.gws_dense_fwd(x, w, y, bias=b, act=act, residual=r, z=z, w_is_nk=nk)
    (wz, wy), (tz, ty) = ref.dense_fwd(x, w, nk, b, act, r0 if in_place else r)
    assert_within(y, wy, ty, ("y", M, K, N, nk, act))
    if keep:
        assert_within(z, wz, tz, ("z", M, K, N, nk, act))
        assert (zwhole[:, N:] == 7).all()
    if whole is not None:
        assert (whole[:, N:] == 7).all()


def check_bwd(M, D, F, nk, act, h=True, db=True, pad=0, alias=None):
    dy, wd = rand(1, M, D, 1e-2, D + pad), (rand(2, D, F, 0.05, F + pad) if nk else rand(2, F, D, 0.05, D + pad))
    z = rand(3, M, F, 1.5, F + 2 * pad)
    z0 = z.clone()
    dz, whole = (z, None) if alias == "dz" else room(M, F, F + pad)
    hh, hwhole = (z, None) if alias == "h" else room(M, F, F + 3 * pad) if h else (None, None)
    dbias = torch.full((F,), math.nan, device=DEV) if db else None
    ws = torch.full((gws.gws_dense_bwd_workspace_bytes(M, F) // 4,), math.nan, device=DEV) if db else None
    gws.gws_dense_bwd(dy, wd, z, dz, act, h=hh, dbias=dbias, workspace=ws, w_is_nk=nk)
    dh, eh = gated_ref.product(dy, wd, not nk)
    want, tol = ref.dense_bwd(dh, eh, z0, act)
    assert_within(dz, want[0], tol[0], ("dz", M, D, F, nk, act))
    if h:
        assert_within(hh, want[1], tol[1], ("h", M, D, F, nk, act))
    if db:
        assert_within(dbias, want[2], tol[2], ("db", M, D, F, nk, act))
    for buf in (whole, hwhole):
        if buf is not None:
            assert (buf[:, F:] == 7).all()


SMALL = [(1, 32, 32), (1, 64, 32), (3, 96, 160), (16, 64, 64), (17, 128, 96), (33, 160, 224), (65, 32, 64), (129, 96, 288), (200, 352, 320)]


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("nk", [False, True])
@pytest.mark.parametrize("M,K,N", SMALL)
def test_forward(M, K, N, nk, act):
    check_fwd(M, K, N, nk, act, pad=8 if M % 2 else 0)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("nk", [False, True])
@pytest.mark.parametrize("M,D,F", SMALL)
def test_backward(M, D, F, nk, act):
    check_bwd(M, D, F, nk, act, pad=8 if M % 2 else 0)


@pytest.mark.parametrize("bias,residual,keep", [(a, b, c) for a in (0, 1) for b in (0, 1) for c in (0, 1)])
def test_parts_of_the_epilogue(bias, residual, keep):
    for M, K, N in ((5, 64, 64), (130, 96, 160)):
        check_fwd(M, K, N, True, gws.ACT_GELU_TANH, bias, residual, keep)
        check_fwd(M, K, N, False, gws.ACT_NONE, bias, residual, keep)


def test_parts_of_the_backward_pass():
    for h in (False, True):
        for db in (False, True):
            check_bwd(70, 64, 96, True, gws.ACT_SILU, h, db)
            check_bwd(9, 64, 96, False, gws.ACT_GELU_TANH, h, db)
    # no activation, no Z
    dy, wd, dz = rand(1, 40, 64), rand(2, 64, 96), room(40, 96)[0]
    gws.gws_dense_bwd(dy, wd, None, dz, w_is_nk=True)
    dh, eh = gated_ref.product(dy, wd, False)
    assert_within(dz, dh, eh + ref.BF16 * dh.abs(), "dz")


@pytest.mark.parametrize("M,K,N", [(8, 64, 96), (300, 64, 64), (1000, 128, 256)])
def test_in_place(M, K, N):
    for nk in (False, True):
        check_fwd(M, K, N, nk, gws.ACT_SILU, in_place=True)
        check_bwd(M, K, N, nk, gws.ACT_SILU, alias="dz")
        check_bwd(M, K, N, nk, gws.ACT_GELU_TANH, alias="h")


@pytest.mark.parametrize("M,F", [(1, 8), (5, 64), (31, 264), (100, 1000), (1021, 520), (5000, 96)])
@pytest.mark.parametrize("act", ACTS)
def test_backward_from_dh(M, F, act):
    ld = F + 16
    dh, z = rand(1, M, F, 1e-2, ld), rand(2, M, F, 1.5, F + 8)
    (dz, whole), h, db = room(M, F, F + 8), room(M, F)[0], torch.full((F,), math.nan, device=DEV)
    ws = torch.full((gws.gws_dense_bwd_workspace_bytes(M, F) // 4,), math.nan, device=DEV)
    gws.gws_dense_bwd_h(dh, z, dz, act, h=h, dbias=db, workspace=ws)
    want, tol = ref.dense_bwd(dh.double(), torch.zeros_like(dh, dtype=torch.float64), z, act)
    for got, w, t, name in zip((dz, h, db), want, tol, ("dz", "h", "db")):
        assert_within(got, w, t, name)
    assert (whole[:, F:] == 7).all()
    same = torch.nn.functional.pad(dh, (0, 16))[:, :F]
    gws.gws_dense_bwd_h(same, z, same, act)
    assert torch.equal(same, dz)
    if act == gws.ACT_NONE:   # the sum alone
        db2 = torch.full((F,), math.nan, device=DEV)
        gws.gws_dense_bwd_h(dh, None, None, dbias=db2, workspace=ws)
        assert torch.equal(db2, db)


def test_no_rows():
    x = torch.zeros(0, 64, dtype=torch.bfloat16, device=DEV)
    w, db = rand(1, 64, 64), torch.full((64,), 3.0, device=DEV)
    gws.gws_dense_fwd(x, w, x, act=gws.ACT_SILU)
    gws.gws_dense_bwd(x, w, x, x, gws.ACT_SILU, dbias=db)
    assert (db == 0).all()
    db.fill_(3.0)
    gws.gws_dense_bwd_h(x, None, None, dbias=db)
    assert (db == 0).all()


def test_without_an_epilogue_it_is_the_plain_product():
    for M, K, N in ((1, 2048, 512), (100, 96, 224), (1021, 768, 768), (2048, 512, 1024)):
        for nk in (False, True):
            x, w, y, y2 = rand(1, M, K), weight(2, K, N, nk), room(M, N)[0], room(M, N)[0]
            gws.gws_dense_fwd(x, w, y, w_is_nk=nk)
            gws.gws_gemm_bf16(x, w, y2, w_is_nk=nk)
            assert torch.equal(y, y2)


def test_values_at_the_edge_of_the_numbers():
    """Activations of very large, infinite and NaN sums; rows of them stay by themselves."""
    M, K, N = 70, 64, 64
    w = torch.eye(64, dtype=torch.bfloat16, device=DEV)
    x = torch.zeros(M, K, dtype=torch.bfloat16, device=DEV)
    x[:, 0] = torch.linspace(-30, 30, M, device=DEV).bfloat16()
    x[1, 1], x[2, 1], x[3, 1], x[4, 1] = 1e30, -1e30, 3e38, -3e38
    x[5, 2] = math.nan
    for act in ACTS:
        y, z = room(M, N)[0], room(M, N)[0]
        gws.gws_dense_fwd(x, w, y, act=act, z=z)
        (wz, wy), (tz, ty) = ref.dense_fwd(x, w, False, None, act, None)
        good = [i for i in range(M) if i != 5]
        assert_within(y[good], wy[good].clamp(-3.39e38, 3.39e38), ty[good], act)
        assert torch.isnan(y[5, 2])
        dh, dz, h = torch.ones(M, N, dtype=torch.bfloat16, device=DEV), room(M, N)[0], room(M, N)[0]
        gws.gws_dense_bwd_h(dh, z, dz, act, h=h)
        want, tol = ref.dense_bwd(dh.double(), torch.zeros(M, N, dtype=torch.float64, device=DEV), z, act)
        assert not torch.isnan(dz[good]).any() and torch.isnan(h[5, 2])
        small = [i for i in good if i > 5]
        assert_within(dz[small], want[0][small], tol[0][small] + 1e-37, act)


def test_repeated_calls_give_the_same_bits():
    M, D, F = 700, 256, 512
    dy, wd, z = rand(1, M, D), rand(2, F, D, 0.05), rand(3, M, F)
    ws = torch.empty(gws.gws_dense_bwd_workspace_bytes(M, F), dtype=torch.uint8, device=DEV)
    first = None
    for _ in range(4):
        dz, db = room(M, F)[0], torch.zeros(F, device=DEV)
        gws.gws_dense_bwd(dy, wd, z, dz, gws.ACT_SILU, dbias=db, workspace=ws)
        first = first or (dz, db)
        assert torch.equal(first[0], dz) and torch.equal(first[1], db)
