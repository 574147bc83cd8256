"""The gated feed-forward block and the 8-bit form of activations in 64 bits, for the tests: plain torch from the definitions,
nothing of the library.  Tensors may be on any device."""
import math

import torch

SILU, GELU = 0, 1
C, K3 = math.sqrt(2.0 / math.pi), 0.044715
ULP = 2.0 ** -24          # half a unit of fp32 at 1
BF16 = 2.0 ** -8          # covers one rounding to BF16 (half a unit, 2^-9) and what is lost beside it


def gate(act, g):
    """a(g) and a'(g) of a float64 tensor."""
    if act == SILU:
        q = torch.sigmoid(g)
        return g * q, q * (1.0 + g * torch.sigmoid(-g))
    t = torch.tanh(C * (g + K3 * g ** 3))
    return 0.5 * g * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * C * (1.0 + 3.0 * K3 * g * g)


def product(x, w, transposed):
    """x * w (x * w^T) in 64 bits, and the bound on what fp32 sums of any order lose of it: K 2^-24 sum |x w|."""
    a, b = x.double(), w.double()
    if transposed:
        b = b.t().contiguous()
    return a @ b, a.shape[1] * ULP * (a.abs() @ b.abs())


def pow2(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def blocks(C):
    return torch.arange(C) // 32


def scale_bytes(v):
    """xscale of float64 v [M x C], by brute force over the exponents: the smallest X with max / X rounding to at most 448, from 2^-117
    to 2^119 (beyond, values saturate at 448 X)."""
    M, C = v.shape
    nb = -(-C // 32)
    pad = torch.zeros(M, nb * 32, dtype=torch.float64, device=v.device)
    pad[:, :C] = v.abs()
    top = pad.reshape(M, nb, 32).amax(dim=2)
    out = torch.full((M, nb), 246, dtype=torch.int64, device=v.device)
    for byte in range(246, 9, -1):
        out = torch.where(top <= 464.0 * 2.0 ** (byte - 127), torch.full_like(out, byte), out)
    out = torch.where(top == 0, torch.full_like(out, 127), out)
    bad = ~torch.isfinite(pad.reshape(M, nb, 32)).all(dim=2)
    return torch.where(bad, torch.full_like(out, 255), out)


def code_table(device):
    """Value of every E4M3 code, from the fields of the byte."""
    c = torch.arange(256, device=device)
    e, m = (c >> 3) & 15, (c & 7).double()
    v = torch.where(e == 0, m / 512.0, (8.0 + m) * pow2(e - 10))
    v[(c & 127) == 127] = math.nan
    return torch.where(c >= 128, -v, v)


def decode(codes, xscale):
    v = code_table(codes.device)[codes.view(torch.uint8).long()]
    s = xscale.view(torch.uint8).long()
    x = torch.where(s == 255, torch.full(s.shape, math.nan, dtype=torch.float64, device=s.device), pow2(s - 127))
    return v * x[:, blocks(codes.shape[1]).to(codes.device)]


def encode(v):
    """Codes and xscale of float64 v: the nearest of all 256 values, the even code of two that are equally near; beyond the largest, that one."""
    xs = scale_bytes(v)
    C = v.shape[1]
    b = blocks(C).to(v.device)
    nan = (xs == 255)[:, b]
    w = torch.where(nan, torch.zeros_like(v), v) * pow2(127 - torch.where(xs == 255, torch.full_like(xs, 127), xs))[:, b]
    mags = code_table(v.device)[:127]
    hi = torch.searchsorted(mags, w.abs()).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    dl, dh = w.abs() - mags[lo], mags[hi] - w.abs()
    code = torch.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    code = torch.where(torch.signbit(w), code + 128, code)
    return torch.where(nan, torch.full_like(code, 127), code).to(torch.uint8), xs.to(torch.uint8)


def assert_within(got, ref, tol, what):
    got, ref = got.double(), ref.double()
    nan = torch.isnan(ref)
    assert torch.equal(torch.isnan(got), nan), (what, "NaN elsewhere")
    inf = torch.isinf(ref)
    assert torch.equal(got[inf], ref[inf]), (what, "infinity elsewhere")
    err = torch.where(nan | inf, torch.zeros_like(ref), (got - ref).abs())
    bad = err > tol
    assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[:4].tolist(), got[bad][:4].tolist(), ref[bad][:4].tolist(), (err / tol)[bad].max().item())


def assert_kept(codes, xscale, v, ev, what):
    """Codes of fp32 sums that are within ev of v: the scale is one of a sum's in that range, the value as near as its spacing allows."""
    lo, hi = scale_bytes((v.abs() - ev).clamp(min=0)), scale_bytes(v.abs() + ev)
    xs = xscale.view(torch.uint8).long()
    assert ((xs >= lo) & (xs <= hi)).all(), (what, "scale")
    x = pow2(xs - 127)[:, blocks(v.shape[1]).to(v.device)]
    spacing = torch.maximum(pow2(torch.frexp(v.abs() + ev)[1].long() - 4), x * 2.0 ** -9)   # of E4M3 at the value
    assert_within(decode(codes, xscale), v, 0.5 * spacing + ev, what)
