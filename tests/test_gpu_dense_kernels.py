"""Every kernel that a call of the dense layer may take, by sizes for which it is the one (gws_dense_form): tiles cut by the
edges of the result, K of whole and half steps, both layouts of the weight."""
import ctypes
import math

import pytest
import torch

import gated_ref
import layer_ref as ref
import paper_2505_11170_amd as gws
from gated_ref import assert_within
from gpu_util import DEV, ensure_built
from paper_2505_11170_amd import binding
from test_gpu_dense import check_bwd, check_fwd, weight
from test_gpu_gated import rand, room
from test_gpu_norm import vec

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_built()


# weight stored [N x K], (rows, columns of a tile, workgroups that fetch the weight, tiles in parts), M, K, N
STREAM = [
    (False, (8, 32, 0, 0), 1, 96, 32), (False, (8, 32, 2, 0), 4, 512, 2144), (False, (8, 32, 3, 0), 4, 672, 1568),
    (False, (16, 32, 0, 0), 9, 96, 32), (False, (16, 32, 2, 0), 12, 512, 2080), (False, (16, 32, 3, 0), 14, 1760, 608),
    (False, (32, 32, 0, 0), 17, 96, 32), (False, (32, 32, 0, 1), 33, 64, 512), (False, (32, 32, 2, 0), 18, 608, 2112), (False, (32, 32, 2, 1), 51, 896, 1216),
    (False, (32, 32, 3, 1), 40, 1312, 832), (False, (32, 64, 0, 0), 1064, 96, 256), (False, (32, 64, 0, 1), 292, 64, 832),
    (False, (64, 64, 0, 0), 1749, 96, 288), (False, (64, 64, 0, 1), 820, 64, 608), (False, (128, 64, 0, 0), 3418, 64, 288), (False, (128, 64, 0, 1), 582, 96, 1664),
    (True, (8, 8, 0, 0), 1, 2080, 32), (True, (8, 8, 0, 1), 3, 2048, 256), (True, (8, 16, 0, 0), 1, 64, 32), (True, (8, 16, 0, 1), 2, 96, 512),
    (True, (8, 32, 0, 1), 1, 96, 4224), (True, (16, 8, 0, 0), 12, 2400, 32), (True, (16, 8, 0, 1), 11, 2304, 256), (True, (16, 16, 0, 0), 9, 96, 32),
    (True, (16, 16, 0, 1), 14, 64, 512), (True, (16, 32, 0, 1), 10, 96, 4192), (True, (32, 32, 0, 0), 18, 96, 32), (True, (32, 32, 0, 1), 102, 64, 256),
    (True, (32, 32, 1, 0), 17, 1376, 768), (True, (32, 32, 1, 1), 18, 896, 1184), (True, (32, 64, 0, 0), 1819, 96, 160), (True, (32, 64, 0, 1), 194, 64, 1216),
    (True, (64, 64, 0, 0), 2814, 64, 160), (True, (64, 64, 0, 1), 260, 96, 1856), (True, (128, 64, 0, 1), 1238, 96, 800)]
MIDDLE = [(False, 96, 514, 64, 3392), (False, 96, 389, 96, 4160), (False, 128, 1036, 64, 2720), (False, 128, 771, 96, 3488), (True, 96, 396, 64, 4288),
          (True, 96, 392, 96, 4224), (True, 128, 516, 64, 4928), (True, 128, 776, 96, 3616)]
OTHERS = [(False, gws.GEMM_LARGE_EDGE, 3717, 448, 3360), (False, gws.GEMM_LARGE_EDGE, 3593, 480, 3424), (True, gws.GEMM_LARGE_EDGE, 3631, 384, 3616),
          (True, gws.GEMM_LARGE_EDGE, 2404, 544, 4832), (False, gws.GEMM_NARROW, 2966, 320, 2784), (False, gws.GEMM_NARROW, 3276, 288, 2464), (True, gws.GEMM_NARROW, 3876, 320, 2112),
          (True, gws.GEMM_NARROW, 2136, 288, 3872), (False, gws.GEMM_LARGE, 4096, 192, 4096), (True, gws.GEMM_LARGE, 4096, 448, 4096),
          (False, gws.DENSE_SHARED, 782, 64, 4800), (False, gws.DENSE_SHARED, 781, 96, 4768), (True, gws.DENSE_SHARED, 906, 64, 4128), (True, gws.DENSE_SHARED, 769, 96, 4832),
          (True, gws.DENSE_SHARED, 1118, 352, 4864), (False, gws.DENSE_SHARED, 2381, 288, 2528), (False, gws.GEMM_ANY_SHAPE, 129, 32, 64)]


def form_of(M, K, N, nk):
    """The one kernel of the forward and of the backward call, whose weight lies the other way round."""
    f = gws.gws_dense_form(gws.DENSE_FWD, M, K, N, w_is_nk=nk)
    assert f == gws.gws_dense_form(gws.DENSE_BWD, M, K, N, w_is_nk=not nk)
    return f


def both(M, K, N, nk, pad=0):
    for act, parts in ((gws.ACT_GELU_TANH, dict(keep=True)), (gws.ACT_NONE, dict(residual=False, keep=False)), (gws.ACT_SILU, dict(bias=False))):
        check_fwd(M, K, N, nk, act, pad=pad, **parts)
    # the product of the backward pass has the weight the other way round
    for act, parts in ((gws.ACT_SILU, {}), (gws.ACT_GELU_TANH, dict(h=False)), (gws.ACT_NONE, dict(db=False))):
        check_bwd(M, K, N, not nk, act, pad=pad, **parts)


@pytest.mark.parametrize("nk,tile,M,K,N", STREAM)
def test_few_rows_or_tiles(nk, tile, M, K, N):
    assert form_of(M, K, N, nk) == gws.GEMM_STREAM and gws.gws_gemm_stream_tile(M, K, N, nk) == tile
    both(M, K, N, nk)


@pytest.mark.parametrize("nk,cols,M,K,N", MIDDLE)
def test_middle_tiles(nk, cols, M, K, N):
    assert form_of(M, K, N, nk) == gws.GEMM_MIDDLE and gws.gws_gemm_tile(M, K, N, nk) == (128, cols)
    both(M, K, N, nk)


@pytest.mark.parametrize("nk,form,M,K,N", OTHERS)
def test_large_tiles_and_others(nk, form, M, K, N):
    assert form_of(M, K, N, nk) == form
    both(M, K, N, nk)


@pytest.mark.parametrize("M,K,N,nk", [(582, 96, 1664, False), (389, 96, 4160, False), (516, 64, 4928, True), (2404, 544, 4832, True), (3276, 288, 2464, False), (769, 96, 4832, True)])
def test_matrices_in_wider_buffers(M, K, N, nk):
    both(M, K, N, nk, pad=8)


@pytest.mark.parametrize("M,K,N", [(3, 2048, 256), (102, 64, 256), (771, 96, 3488), (4096, 192, 4096), (3276, 288, 2464), (781, 96, 4768)])
def test_in_place(M, K, N):
    for nk in (False, True):
        check_fwd(M, K, N, nk, gws.ACT_SILU, in_place=True)
        check_bwd(M, K, N, not nk, gws.ACT_SILU, alias="dz")
        check_bwd(M, K, N, not nk, gws.ACT_GELU_TANH, alias="h")


@pytest.mark.parametrize("M,K,N", [(1, 2080, 64), (40, 1312, 832), (771, 96, 3488), (2404, 544, 4832), (4096, 192, 4096), (3276, 288, 2464), (781, 96, 4768)])
def test_results_do_not_change_from_call_to_call_or_with_the_rows_beside(M, K, N):
    """Rows of NaN leave the others as they are; the bias gradient is the same bits every time."""
    x, w, b, r = rand(1, M, K), weight(2, K, N, True), vec(3, N), rand(4, M, N)
    y, z = room(M, N)[0], room(M, N)[0]
    gws.gws_dense_fwd(x, w, y, bias=b, act=gws.ACT_SILU, residual=r, z=z, w_is_nk=True)
    ws, first = torch.empty(gws.gws_dense_bwd_workspace_bytes(M, N), dtype=torch.uint8, device=DEV), None
    for _ in range(3):
        dz, h, db = room(M, N)[0], room(M, N)[0], torch.zeros(N, device=DEV)
        gws.gws_dense_bwd(x, w, z, dz, gws.ACT_SILU, h=h, dbias=db, workspace=ws)
        first = first or (dz, h, db)
        assert all(torch.equal(a, c) for a, c in zip(first, (dz, h, db)))
    if M > 1:
        bad = M // 2
        x2, z2 = x.clone(), z.clone()
        x2[bad] = math.nan
        y2, dz2 = room(M, N)[0], room(M, N)[0]
        good = [i for i in range(M) if i != bad]
        gws.gws_dense_fwd(x2, w, y2, bias=b, act=gws.ACT_SILU, residual=r, z=z2, w_is_nk=True)
        assert torch.equal(y2[good], y[good]) and torch.equal(z2[good], z[good]) and torch.isnan(y2[bad]).all()
        gws.gws_dense_bwd(x2, w, z, dz2, gws.ACT_SILU)
        assert torch.equal(dz2[good], first[0][good])


def test_large_leading_dimensions():
    """Results whose rows lie further apart than the kernels' lane offsets reach, and than 4 GiB of elements together."""
    M, K, N, ld = 20, 64, 64, 1 << 28                # 20 rows 512 MiB apart
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("no room")
    buf = torch.empty(M, ld, dtype=torch.bfloat16, device=DEV)
    x, w, b = rand(1, M, K), weight(2, K, N, True), vec(3, N)
    y, z, r = buf[:, :N], buf[:, 64:64 + N], buf[:, 256:256 + N]
    r.copy_(rand(4, M, N))
    gws.gws_dense_fwd(x, w, y, bias=b, act=gws.ACT_SILU, residual=r, z=z, w_is_nk=True)
    (wz, wy), (tz, ty) = ref.dense_fwd(x, w, True, b, gws.ACT_SILU, r)
    assert_within(y, wy, ty, "y")
    assert_within(z, wz, tz, "z")
    dz, db = buf[:, 512:512 + N], torch.zeros(N, device=DEV)
    ws = torch.empty(gws.gws_dense_bwd_workspace_bytes(M, N), dtype=torch.uint8, device=DEV)
    dy, wd = rand(5, M, K, 1e-2), rand(6, N, K, 0.05)
    gws.gws_dense_bwd(dy, wd, z, dz, gws.ACT_SILU, dbias=db, workspace=ws)
    want, tol = ref.dense_bwd(*gated_ref.product(dy, wd, True), z, gws.ACT_SILU)
    assert_within(dz, want[0], tol[0], "dz")
    assert_within(db, want[2], tol[2], "db")
    # and within those offsets, past 4 GiB
    ld = (1 << 28) - 8
    buf = buf.view(-1)[:M * ld].view(M, ld)
    y, z, r = buf[:, :N], buf[:, 64:64 + N], buf[:, 256:256 + N]
    r.copy_(rand(4, M, N))
    gws.gws_dense_fwd(x, w, y, bias=b, act=gws.ACT_SILU, residual=r, z=z, w_is_nk=True)
    assert_within(y, wy, ty, "y")


@pytest.mark.parametrize("form,M,K,N", [(gws.GEMM_LARGE, 14336, 1024, 6400), (gws.GEMM_LARGE_EDGE, 14300, 512, 6432), (gws.GEMM_NARROW, 15663, 1696, 6208)])
def test_results_that_go_past_the_caches(form, M, K, N):
    """Y, dZ and H of more than 172 MB."""
    for nk in (True, False):
        assert M * N * 2 >= 172 << 20 and form_of(M, K, N, nk) == form
        check_fwd(M, K, N, nk, gws.ACT_GELU_TANH)
        check_bwd(M, K, N, not nk, gws.ACT_SILU)


@pytest.mark.parametrize("M,K,N", [(1021, 2048, 768), (4096, 192, 4096)])
def test_leading_dimensions_of_what_is_left_out_say_nothing(M, K, N):
    """NULL residual, Z and H: whatever stands beside them, the kernel and the bits are the same."""
    lib, stream = binding.load_library(), torch.cuda.current_stream().cuda_stream
    x, w, b, z = rand(1, M, K), weight(2, K, N, True), vec(3, N), rand(4, M, N)
    ws = torch.empty(gws.gws_dense_bwd_workspace_bytes(M, N), dtype=torch.uint8, device=DEV)
    nothing, first = None, None
    for ld in (0, -1, 1 << 30, (1 << 28) + 8):
        y, dz, db = room(M, N)[0], room(M, N)[0], torch.zeros(N, device=DEV)
        e = binding._CEpilogue(b.data_ptr(), gws.ACT_NONE, nothing, ld, nothing, ld)
        assert lib.gws_dense_fwd(x.data_ptr(), M, K, K, w.data_ptr(), N, K, 1, y.data_ptr(), N, ctypes.byref(e), stream) == 0
        # with Z; without; from dH, where only the sum is wanted
        bwd = lambda z, ldz, act: lib.gws_dense_bwd(x.data_ptr(), M, K, K, w.data_ptr(), N, K, 0, act, z, ldz, dz.data_ptr(), N, nothing, ld, db.data_ptr(), ws.data_ptr(),  # noqa: E731
                                                    ws.nbytes, stream)
        out = [y]
        for args in ((z.data_ptr(), N, gws.ACT_SILU), (nothing, ld, gws.ACT_NONE)):
            assert bwd(*args) == 0
            out += [dz.clone(), db.clone()]
        assert lib.gws_dense_bwd_h(z.data_ptr(), M, N, N, gws.ACT_NONE, nothing, ld, nothing, ld, nothing, ld, db.data_ptr(), ws.data_ptr(), ws.nbytes, stream) == 0
        out.append(db)
        first = first or out
        assert all(torch.equal(p, q) for p, q in zip(first, out)), ld


def test_grids_of_more_than_32_bits_of_threads():
    """More than 2^24 of the smallest tiles: every row is written, and the bias gradient has them all."""
    if torch.cuda.mem_get_info()[0] < 190 << 30:
        pytest.skip("no room")
    more_than_32_bits_of_threads()
    torch.cuda.empty_cache()       # 170 GB, which other tests have a use for


def more_than_32_bits_of_threads():
    M, K, N = (1 << 25) + 70, 32, 2048
    assert form_of(M, K, N, True) == gws.GEMM_ANY_SHAPE
    marks = [0, 63, 64, (1 << 21) - 1, 1 << 21, (1 << 24) + 5, (1 << 25) - 1, 1 << 25, M - 1]
    x, w = torch.zeros(M, K, dtype=torch.bfloat16, device=DEV), torch.randint(1, 100, (N, K), generator=torch.Generator(device=DEV).manual_seed(1), device=DEV).bfloat16()
    for i, r in enumerate(marks):
        x[r, i] = 1.0
    y, b = torch.full((M, N), 7, dtype=torch.bfloat16, device=DEV), torch.zeros(N, device=DEV)

    def rows_of_w():
        assert all(torch.equal(y[r], w[:, i]) for i, r in enumerate(marks))
        y[marks] = 0
        assert not any(bool((y[r:r + (1 << 21)] != 0).any()) for r in range(0, M, 1 << 21))

    gws.gws_dense_fwd(x, w, y, bias=b, w_is_nk=True)
    rows_of_w()
    y.fill_(7)
    ws = torch.empty(gws.gws_dense_bwd_workspace_bytes(M, N), dtype=torch.uint8, device=DEV)
    gws.gws_dense_bwd(x, w, None, y, dbias=b, workspace=ws)
    rows_of_w()
    assert torch.equal(b, w[:, :len(marks)].float().sum(1))      # whole numbers: exact


@pytest.mark.parametrize("form,M,K,N", [(gws.GEMM_LARGE_EDGE, 14300, 1056, 6432), (gws.DENSE_SHARED, 117567, 1056, 800), (gws.GEMM_NARROW, 73332, 992, 1344)])
def test_results_that_go_past_the_caches_where_their_readers_wait_for_the_products(form, M, K, N):
    """Of the other forms those that the backward pass too takes past the caches (D of 1024 and more), and one of shorter products, whose backward pass does not."""
    for nk in (True, False):
        assert M * N * 2 >= 172 << 20 and form_of(M, K, N, nk) == form
        check_fwd(M, K, N, nk, gws.ACT_SILU)
        check_bwd(M, K, N, not nk, gws.ACT_GELU_TANH)
