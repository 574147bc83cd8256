"""Activations in 8 bits: gws_act8_encode and gws_act8_decode bit for bit against the definition."""
import math

import pytest
import torch

import gated_ref as ref
import paper_2505_11170_amd as gws
from gpu_util import DEV, ensure_built

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_built()


def buffers(M, C, ldc=None, lds=None):
    nb = -(-C // 32)
    codes = torch.full((M, ldc or -(-C // 8) * 8), 0xA5, dtype=torch.uint8, device=DEV)
    xs = torch.full((M, lds or nb), 0xA5, dtype=torch.uint8, device=DEV)
    return codes, xs, gws.Act8(codes[:, :C], xs[:, :nb])


def padded(v, ld=None):
    M, C = v.shape
    x = torch.full((M, ld or -(-C // 8) * 8), math.nan, dtype=torch.bfloat16, device=DEV)
    x[:, :C] = v.to(DEV)
    return x, x[:, :C]


def check(v, ldc=None, lds=None, ldx=None):
    M, C = v.shape
    nb = -(-C // 32)
    _, x = padded(v, ldx)
    codes, xs, a = buffers(M, C, ldc, lds)
    gws.gws_act8_encode(x, a)
    torch.cuda.synchronize()
    rc, rs = ref.encode(x.double())
    assert torch.equal(a.xscale, rs), (a.xscale != rs).nonzero()[:4]
    assert torch.equal(a.codes, rc), (a.codes != rc).nonzero()[:4]
    assert (codes[:, C:] == 0xA5).all() and (xs[:, nb:] == 0xA5).all()      # past a row's data nothing is written
    back, y = padded(torch.zeros(M, C, dtype=torch.bfloat16), ldx)
    gws.gws_act8_decode(a, y)
    torch.cuda.synchronize()
    want = ref.decode(a.codes, a.xscale)
    assert torch.equal(torch.isnan(y), torch.isnan(want))
    ok = ~torch.isnan(want)
    assert torch.equal(y.double()[ok], want[ok])                           # exact
    assert torch.equal(torch.signbit(y)[ok], torch.signbit(want)[ok])      # zeros keep their sign
    assert torch.isnan(back[:, C:]).all()


@pytest.mark.parametrize("M,C", [(1, 1), (1, 32), (3, 31), (7, 33), (1, 5632), (301, 1000), (64, 96), (33, 4099), (2049, 40)])
def test_random_values(M, C):
    gen = torch.Generator().manual_seed(M * 10007 + C)
    v = torch.randn(M, C, generator=gen) * torch.exp(4.0 * torch.randn(M, 1, generator=gen))
    v[:, ::7] *= 64.0
    v[M // 2] = 0.0
    check(v.bfloat16())


@pytest.mark.parametrize("shift", [-120, -109, -100, 0, 100, 119])
def test_every_value_under_every_kind_of_largest(shift):
    # each row: a block whose largest magnitude is 2^shift (1 + m / 128), and values of all binades below it
    gen = torch.Generator().manual_seed(5)
    m = torch.arange(128)
    v = torch.zeros(128 * 8, 32, dtype=torch.float64)
    v[:, 0] = (1.0 + m.repeat(8) / 128.0) * 2.0 ** shift
    v[:, 1:] = torch.ldexp(1.0 + torch.randint(0, 128, (128 * 8, 31), generator=gen) / 128.0, torch.randint(-20, 0, (128 * 8, 31), generator=gen)).double() * 2.0 ** shift
    v[:, 1::2] *= -1.0
    check(v.bfloat16())


def test_ties_and_every_bf16_value():
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    fine = bits[torch.isfinite(bits)]
    check(torch.cat([fine, fine.new_zeros(-fine.numel() % 32)]).reshape(-1, 32))          # 32 neighbouring patterns a block
    # all values of a block whose scale is 2^-8 x 2^e: ties of every code
    v = torch.cat([torch.full((256, 1), 1.8125), torch.arange(256).reshape(256, 1) * 2.0 ** -8, torch.arange(256).reshape(256, 1) * 2.0 ** -18], dim=1)
    check(v.bfloat16())


def test_nan_and_infinity_stay_in_their_block():
    v = torch.randn(5, 100, generator=torch.Generator().manual_seed(2))
    v[1, 40], v[2, 0], v[2, 99], v[3, 95] = math.nan, math.inf, -math.inf, math.nan
    v = v.bfloat16()
    check(v)
    _, x = padded(v)
    _, _, a = buffers(5, 100)
    gws.gws_act8_encode(x, a)
    _, y = padded(torch.zeros_like(v))
    gws.gws_act8_decode(a, y)
    torch.cuda.synchronize()
    want = torch.zeros(5, 100, dtype=torch.bool)
    want[1, 32:64] = want[2, 0:32] = want[2, 96:] = want[3, 64:96] = True
    assert torch.equal(torch.isnan(y).cpu(), want)


def test_wide_rows_of_larger_buffers_and_another_stream():
    v = torch.randn(70, 200, generator=torch.Generator().manual_seed(3)).bfloat16()
    check(v, ldc=4096, lds=77, ldx=1000)
    s = torch.cuda.Stream()
    _, x = padded(v)
    codes, xs, a = buffers(70, 200)
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        gws.gws_act8_encode(x, a)
    s.synchronize()
    rc, rs = ref.encode(x.double())
    assert torch.equal(a.codes, rc) and torch.equal(a.xscale, rs)


def test_offsets_beyond_32_bits():
    # rows 64 KiB apart: the last ones lie past 4 GiB in x, and past it in elements of nothing smaller
    M, C, ld = 66000, 40, 32768 + 8
    x = torch.empty(M, ld, dtype=torch.bfloat16, device=DEV)
    v = torch.randn(M, C, device=DEV, generator=torch.Generator(device=DEV).manual_seed(4)).bfloat16()
    x[:, :C] = v
    codes = torch.empty(M, 65536 + 8, dtype=torch.uint8, device=DEV)
    xs = torch.empty(M, 2, dtype=torch.uint8, device=DEV)
    a = gws.Act8(codes[:, :C], xs)
    gws.gws_act8_encode(x[:, :C], a)
    torch.cuda.synchronize()
    rc, rs = ref.encode(v.double())
    assert torch.equal(a.codes, rc) and torch.equal(xs, rs)
    x.zero_()
    gws.gws_act8_decode(a, x[:, :C])
    torch.cuda.synchronize()
    assert torch.equal(x[:, :C].double(), ref.decode(rc, rs)) and (x[:, C:64] == 0).all()


def test_empty():
    x = torch.zeros(0, 64, dtype=torch.bfloat16, device=DEV)
    gws.gws_act8_encode(x, gws.Act8(torch.zeros(0, 64, dtype=torch.uint8, device=DEV), torch.zeros(0, 2, dtype=torch.uint8, device=DEV), ldc=64, lds=2))
