"""Layer norm and root-mean-square norm, forward and backward, against 64 bits (bounds: layer_ref.py)."""
import math

import pytest
import torch

import layer_ref as ref
import paper_2505_11170_amd as gws
from gated_ref import assert_within
from gpu_util import DEV, ensure_built
from test_gpu_gated import rand, room

pytestmark = pytest.mark.gpu
LAYER, RMS = gws.NORM_LAYER, gws.NORM_RMS


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_built()


def vec(seed, n, mean=0.0, std=1.0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    return mean + std * torch.randn(n, generator=gen, device=DEV)


def ld_of(C, wide=False):
    return -(-C // 8) * 8 + (24 if wide else 0)


def odd_start(v):
    """The same vector from an address that is a multiple of four only."""
    return torch.cat([torch.full((1,), math.nan, device=DEV), v])[1:]


def untouched(whole, C):
    return bool((whole[:, C:] == 7).all())


# one lane's part of a row, a row of each width of kernel and one element to either side, rows that are read again
SIZES = [(1, 1), (3, 7), (1, 2048), (5, 64), (131, 128), (77, 129), (2, 256), (2, 511), (5, 514), (70, 677), (33, 766), (300, 768), (3, 771), (3, 1030), (2, 4101), (2, 16387), (6, 1536), (7, 513), (3, 1025), (1021, 1000), (3, 2047), (9, 2049), (2, 4100), (5, 8192), (3, 8200),
         (2, 16384), (2, 16385), (3, 40003)]


@pytest.mark.parametrize("kind", [LAYER, RMS])
@pytest.mark.parametrize("M,C", SIZES)
def test_forward(M, C, kind):
    wide = C % 2 == 1
    x = rand(M + C, M, C, ld=ld_of(C, wide)) * 2 + 0.5
    x = torch.nn.functional.pad(x, (0, ld_of(C, wide) - C), value=math.nan)[:, :C]
    gamma, beta = odd_start(vec(1, C, 1.0, 0.2)), odd_start(vec(2, C, 0.0, 0.3))
    (y, whole), mean, rstd = room(M, C, ld_of(C) + 8), torch.full((M,), math.nan, device=DEV), torch.full((M,), math.nan, device=DEV)
    gws.gws_norm_fwd(x, y, kind, gamma=gamma, beta=beta, eps=1e-5, mean=mean if kind == LAYER else None, rstd=rstd)
    want, tol = ref.norm_fwd(x, kind, gamma, beta, 1e-5)
    assert_within(y, want[0], tol[0], "y")
    assert_within(rstd, want[2], tol[2], "rstd")
    if kind == LAYER:
        assert_within(mean, want[1], tol[1], "mean")
    assert untouched(whole, C)
    # nothing kept, no gamma, no beta; the same numbers where they are the same
    y2 = room(M, C, ld_of(C))[0]
    gws.gws_norm_fwd(x, y2, kind, gamma=gamma, beta=beta, eps=1e-5)
    assert torch.equal(y2, y)
    gws.gws_norm_fwd(x, y2, kind)
    want, tol = ref.norm_fwd(x, kind, None, None, 1e-5)
    assert_within(y2, want[0], tol[0], "bare")


@pytest.mark.parametrize("kind", [LAYER, RMS])
@pytest.mark.parametrize("M,C", SIZES)
def test_backward(M, C, kind):
    wide = C % 2 == 0
    ld = ld_of(C, wide)
    x, dy, r = rand(1, M, C, 1.5, ld), rand(2, M, C, 1e-3, ld + 8), rand(3, M, C, 1e-3, ld_of(C))
    gamma = odd_start(vec(4, C, 1.0, 0.2))
    xd = x.double()
    mean = xd.mean(1) if kind == LAYER else xd.new_zeros(M)
    rstd = (1.0 / torch.sqrt(((xd - mean[:, None]) ** 2).mean(1) + 1e-5)).float()
    mean = mean.float()
    (dx, whole), dgamma, dbeta = room(M, C, ld_of(C) + 16), torch.full((C,), math.nan, device=DEV), torch.full((C,), math.nan, device=DEV)
    ws = torch.full((gws.gws_norm_bwd_workspace_bytes(M, C) // 4,), math.nan, device=DEV)
    kept = dict(kind=kind, mean=mean if kind == LAYER else None, gamma=gamma)
    gws.gws_norm_bwd(dy, x, dx, rstd, residual=r, dgamma=dgamma, dbeta=dbeta, workspace=ws, **kept)
    want, tol = ref.norm_bwd(dy, x, kind, gamma, mean, rstd, r)
    for got, w, t, name in zip((dx, dgamma, dbeta), want, tol, ("dx", "dgamma", "dbeta")):
        assert_within(got, w, t, name)
    assert untouched(whole, C)
    # one of the two sums alone, none, no residual; the same bits
    one, dx2 = torch.full((C,), math.nan, device=DEV), room(M, C, ld_of(C))[0]
    gws.gws_norm_bwd(dy, x, dx2, rstd, dbeta=one, workspace=ws, residual=r, **kept)
    assert torch.equal(one, dbeta) and torch.equal(dx2, dx)
    gws.gws_norm_bwd(dy, x, dx2, rstd, dgamma=one, workspace=ws, **kept)
    assert torch.equal(one, dgamma)
    want, tol = ref.norm_bwd(dy, x, kind, gamma, mean, rstd, None)
    assert_within(dx2, want[0], tol[0], "without residual")
    gws.gws_norm_bwd(dy, x, dx2, rstd, kind, mean=kept["mean"], workspace=ws if C > 16384 else None)
    want, tol = ref.norm_bwd(dy, x, kind, None, mean, rstd, None)
    assert_within(dx2, want[0], tol[0], "bare")


@pytest.mark.parametrize("M,C", [(20000, 96), (5001, 250), (2100, 400), (2500, 1000), (2049, 1500), (2050, 2048), (1100, 4000), (1100, 6000), (1100, 8000), (600, 9000), (1300, 4000), (1600, 9000), (1000, 1500), (1000, 6000), (200, 30000), (3000, 768), (3001, 701), (2050, 1003)])
def test_many_rows(M, C):
    x, dy = rand(1, M, C, ld=ld_of(C)), rand(2, M, C, 1e-3, ld_of(C))
    y, mean, rstd = room(M, C, ld_of(C))[0], torch.zeros(M, device=DEV), torch.zeros(M, device=DEV)
    gws.gws_norm_fwd(x, y, mean=mean, rstd=rstd)
    want, tol = ref.norm_fwd(x, LAYER, None, None, 1e-5)
    assert_within(y, want[0], tol[0], "y")
    dx, dgamma, dbeta = room(M, C, ld_of(C))[0], torch.zeros(C, device=DEV), torch.zeros(C, device=DEV)
    ws = torch.empty(gws.gws_norm_bwd_workspace_bytes(M, C), dtype=torch.uint8, device=DEV)
    gws.gws_norm_bwd(dy, x, dx, rstd, mean=mean, dgamma=dgamma, dbeta=dbeta, workspace=ws)
    want, tol = ref.norm_bwd(dy, x, LAYER, None, mean, rstd, None)
    for got, w, t, name in zip((dx, dgamma, dbeta), want, tol, ("dx", "dgamma", "dbeta")):
        assert_within(got, w, t, name)
    first = [t.clone() for t in (dx, dgamma, dbeta)]
    for _ in range(3):   # one order of all sums
        gws.gws_norm_bwd(dy, x, dx, rstd, mean=mean, dgamma=dgamma, dbeta=dbeta, workspace=ws)
        assert all(torch.equal(a, b) for a, b in zip(first, (dx, dgamma, dbeta)))


@pytest.mark.parametrize("C", [768, 2048, 3000, 20000])
def test_rows_at_the_edge_of_the_numbers(C):
    """A far common offset, constant rows, zeros, the largest and smallest values; rows of NaN or infinity stay by themselves."""
    x = rand(5, 12, C)
    x[0] = (x[0].float() * 0.5 + 300.0).bfloat16()
    x[1], x[2] = 3.0, 0.0
    x[3] = (x[3].float() * 1e18).bfloat16()
    x[4] = (x[4].float() * 1e-30).bfloat16()
    x[6, C // 2], x[8, C - 1], x[10, 0] = math.nan, math.inf, -math.inf
    for kind in (LAYER, RMS):
        y, mean, rstd = room(12, C)[0], torch.zeros(12, device=DEV), torch.zeros(12, device=DEV)
        gws.gws_norm_fwd(x, y, kind, mean=mean if kind == LAYER else None, rstd=rstd)
        want, tol = ref.norm_fwd(x, kind, None, None, 1e-5)
        good = [i for i in range(12) if i not in (6, 8, 10)]
        assert_within(y[good], want[0][good], tol[0][good], kind)
        assert torch.isnan(y[6]).all() and torch.isnan(y[8, C - 1]) and torch.isnan(y[10, 0])
        assert (y[2] == 0).all() and rstd[2] == torch.tensor(1.0) / torch.sqrt(torch.tensor(1e-5))
        if kind == LAYER:
            assert (y[1] == 0).all()
        dy, dx = rand(6, 12, C), room(12, C)[0]
        dy[4, 1] = math.nan
        bad = (4, 6, 8, 10)
        ws = torch.empty(gws.gws_norm_bwd_workspace_bytes(12, C), dtype=torch.uint8, device=DEV)
        gws.gws_norm_bwd(dy, x, dx, rstd, kind, mean=mean, workspace=ws)
        want, tol = ref.norm_bwd(dy, x, kind, None, mean, rstd, None)
        good = [i for i in range(12) if i not in bad]
        assert_within(dx[good], want[0][good], tol[0][good], kind)
        assert torch.isnan(dx[4]).all() and torch.isnan(dx[6]).all()


@pytest.mark.parametrize("C", [100, 1000, 5000, 17000])
def test_in_place(C):
    M = 37
    x, dy, r = rand(1, M, C, ld=ld_of(C)), rand(2, M, C, ld=ld_of(C)), rand(3, M, C, ld=ld_of(C))
    y, mean, rstd = room(M, C, ld_of(C))[0], torch.zeros(M, device=DEV), torch.zeros(M, device=DEV)
    gws.gws_norm_fwd(x, y, mean=mean, rstd=rstd)
    same = torch.nn.functional.pad(x, (0, ld_of(C) - C))[:, :C]
    gws.gws_norm_fwd(same, same)
    assert torch.equal(same, y)
    ws = torch.empty(gws.gws_norm_bwd_workspace_bytes(M, C), dtype=torch.uint8, device=DEV)
    dx = room(M, C, ld_of(C))[0]
    gws.gws_norm_bwd(dy, x, dx, rstd, mean=mean, residual=r, workspace=ws)
    for k in range(3):
        a = [torch.nn.functional.pad(t, (0, ld_of(C) - C))[:, :C] for t in (dy, x, r)]
        gws.gws_norm_bwd(a[0], a[1], a[k], rstd, mean=mean, residual=a[2], workspace=ws)
        assert torch.equal(a[k], dx)


def test_gradients_against_differences():
    """d(sum of dY y) along random directions of x, gamma and beta, from the 64-bit definition."""
    M, C, h = 6, 200, 1e-4
    for kind in (LAYER, RMS):
        x, dy = rand(1, M, C).double(), rand(2, M, C).double()
        gamma, beta = vec(3, C, 1.0, 0.2).double(), vec(4, C).double()
        f = lambda x, gamma, beta: (ref.norm_fwd(x, kind, gamma, beta, 1e-5)[0][0] * dy).sum()  # noqa: E731
        (_, mean, rstd), _ = ref.norm_fwd(x, kind, gamma, beta, 1e-5)
        dx, dgamma, dbeta = room(M, C)[0], torch.zeros(C, device=DEV), torch.zeros(C, device=DEV)
        ws = torch.empty(gws.gws_norm_bwd_workspace_bytes(M, C), dtype=torch.uint8, device=DEV)
        gws.gws_norm_bwd(dy.bfloat16(), x.bfloat16(), dx, rstd.float(), kind, mean=mean.float(), gamma=gamma.float(), dgamma=dgamma, dbeta=dbeta, workspace=ws)
        for grad, at in ((dx, 0), (dgamma, 1), (dbeta, 2)):
            u = torch.randn(grad.shape, generator=torch.Generator(device=DEV).manual_seed(9), device=DEV).double()
            args = [x, gamma, beta]
            slope = (f(*[a + h * u if i == at else a for i, a in enumerate(args)]) - f(*[a - h * u if i == at else a for i, a in enumerate(args)])) / (2 * h)
            # dX rounded to BF16; a third derivative of order 10 times h^2
            assert abs((grad.double() * u).sum() - slope) <= (ref.BF16 if at == 0 else 1e-5) * (grad.double() * u).abs().sum() + 1e-4


def test_no_rows():
    x, e = torch.zeros(0, 64, dtype=torch.bfloat16, device=DEV), torch.zeros(0, device=DEV)
    gws.gws_norm_fwd(x, x, mean=e, rstd=e)
    dgamma, dbeta = torch.full((64,), 3.0, device=DEV), torch.full((64,), 3.0, device=DEV)
    gws.gws_norm_bwd(x, x, x, e, mean=e, dgamma=dgamma, dbeta=dbeta)
    assert (dgamma == 0).all() and (dbeta == 0).all()


def test_offsets_past_32_bits():
    """Rows that lie beyond 4 GiB of elements of a wide buffer."""
    M, C, ld = 35, 100, 1 << 27                      # 35 x 2^27 elements x 2 bytes: 9.4 GB
    if torch.cuda.mem_get_info()[0] < 30 << 30:
        pytest.skip("no room")
    buf = torch.empty(M, ld, dtype=torch.bfloat16, device=DEV)
    x, y = buf[:, :C], buf[:, 128:128 + C]
    x.copy_(rand(1, M, C))
    gws.gws_norm_fwd(x, y)
    want, tol = ref.norm_fwd(x, LAYER, None, None, 1e-5)
    assert_within(y, want[0], tol[0], "y")


def test_grids_of_more_than_32_bits_of_threads():
    """Four million long rows, in place; a row of half a billion columns with both gradients."""
    if torch.cuda.mem_get_info()[0] < 150 << 30:
        pytest.skip("no room")
    M, C = (1 << 22) + 3, 16392
    x, rstd = torch.zeros(M, C, dtype=torch.bfloat16, device=DEV), torch.full((M,), -1.0, device=DEV)
    marks = [0, 1, (1 << 20) - 1, 1 << 20, (1 << 22) - 1, 1 << 22, M - 1]
    for r in marks:
        x[r] = 3.0
    gws.gws_norm_fwd(x, x, RMS, eps=2.0 ** -20, rstd=rstd)
    ones = torch.zeros(M, dtype=torch.bool, device=DEV)
    ones[marks] = True
    assert torch.equal(x[:, 5] != 0, ones) and torch.equal(x[:, C - 1], ones.bfloat16())      # 3 / sqrt(9 + 2^-20) rounds to 1
    assert bool((rstd[~ones] == 1024.0).all()) and bool(((rstd[ones] * 3.0 - 1.0).abs() < 1e-6).all())
    del x, rstd, ones
    torch.cuda.empty_cache()
    C = (1 << 29) + 40
    x = torch.randint(0, 4, (1, C), dtype=torch.int8, device=DEV).bfloat16()
    dy = torch.randint(-1, 2, (1, C), dtype=torch.int8, device=DEV).bfloat16()
    dx, dgamma, dbeta = torch.empty_like(x), torch.full((C,), 9.0, device=DEV), torch.full((C,), 9.0, device=DEV)
    mean, rstd = torch.tensor([0.25], device=DEV), torch.tensor([2.0], device=DEV)
    ws = torch.empty(gws.gws_norm_bwd_workspace_bytes(1, C), dtype=torch.uint8, device=DEV)
    gws.gws_norm_bwd(dy, x, dx, rstd, kind=LAYER, mean=mean, dgamma=dgamma, dbeta=dbeta, workspace=ws)
    assert torch.equal(dbeta, dy[0].float()) and torch.equal(dgamma, dy[0].float() * (x[0].float() * 2 - 0.5))   # exact in every step


CONSTANTS = [2.0 ** 120, -3e38, 2.0 ** 126, 1e36, 3e38, 255.0, -255 * 2.0 ** 20, 3.0, 2.0 ** -130, 0.0]


@pytest.mark.parametrize("C", [8, 768, 2048, 3000, 20000, 70001])
@pytest.mark.parametrize("eps", [1e-5, 3000.0])
def test_constant_rows(C, eps):
    """Y is beta and rstd 1 / sqrt(eps), also where the row's sum leaves fp32's range or has more bits than fp32 holds."""
    values, n = CONSTANTS, len(CONSTANTS)
    x = rand(7, n + 3, C, 1.0, ld_of(C))
    for i, v in enumerate(values):
        x[i] = v
    x[n, 0] = 2.0 ** 120                                # not constant: a row of N(0, 1) beside 2^120
    gamma, beta = vec(9, C, 1.0, 0.2), vec(10, C)
    y, mean, rstd = room(n + 3, C, ld_of(C))[0], torch.full((n + 3,), math.nan, device=DEV), torch.full((n + 3,), math.nan, device=DEV)
    gws.gws_norm_fwd(x, y, gamma=gamma, beta=beta, eps=eps, mean=mean, rstd=rstd)
    assert torch.equal(mean[:n], x[:n, 0].float())
    alone = 1.0 / math.sqrt(torch.tensor(eps).item())   # of eps as fp32; a root and a quotient, each rounded
    assert bool(((rstd[:n].double() - alone).abs() <= 2 * ref.U * alone).all())
    for i in range(n):
        assert torch.equal(y[i], beta.bfloat16()), values[i]
    want, tol = ref.norm_fwd(x, LAYER, gamma, beta, eps)
    assert_within(y[n:], want[0][n:], tol[0][n:], "y")
    assert_within(rstd[n:], want[2][n:], tol[2][n:], "rstd")


@pytest.mark.parametrize("M,C", [(13, 8), (13, 100), (13, 700), (13, 2000), (13, 3000), (13, 20001), (1300, 8), (1300, 100), (1300, 700), (1300, 2000), (1300, 3000)])
def test_gradients_of_constant_rows(M, C):
    """n is 0 in them, however large mean times rstd: their dX has the row's t alone, and they add nothing to dgamma."""
    n = len(CONSTANTS)
    x, dy = rand(7, M, C, 1.0, ld_of(C)), rand(8, M, C, 1.0, ld_of(C))
    for i, v in enumerate(CONSTANTS):
        x[i] = v
    gamma = vec(9, C, 1.0, 0.2)
    mean = x.double().mean(1)
    rstd = (1.0 / torch.sqrt(((x.double() - mean[:, None]) ** 2).mean(1) + 1e-5)).float()
    mean = mean.float()
    dx, dgamma, dbeta = room(M, C, ld_of(C))[0], torch.zeros(C, device=DEV), torch.zeros(C, device=DEV)
    ws = torch.empty(gws.gws_norm_bwd_workspace_bytes(M, C), dtype=torch.uint8, device=DEV)
    want, tol = ref.norm_bwd(dy, x, LAYER, gamma, mean, rstd, None)
    for _ in range(2):
        gws.gws_norm_bwd(dy, x, dx, rstd, mean=mean, gamma=gamma, dgamma=dgamma, dbeta=dbeta, workspace=ws)
        for got, w, t, name in zip((dx, dgamma, dbeta), want, tol, ("dx", "dgamma", "dbeta")):
            assert_within(got, w, t, name)
        dx = torch.nn.functional.pad(dy, (0, ld_of(C) - C))[:, :C]     # then in place, by the other kernel
        dy = dx
