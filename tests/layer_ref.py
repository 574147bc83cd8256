"""The norms, the dense layer and the AdamW step from their definitions, for the tests: plain torch and numpy, nothing of the library.

Bounds on what fp32 loses, u = 2^-24 (half a unit at 1): a sum whose longest chain of additions is k long is within k u of the sum of its terms' sizes,
a chain of a few operations within a few u, a result rounded once to BF16 within 2^-8 of its size."""
import numpy as np
import torch

import gated_ref

U, BF16, TINY = 2.0 ** -24, 2.0 ** -8, 2.0 ** -126
ARITH = 2.0 ** -16        # of an activation's arithmetic, times 1 + |z| (test_gpu_gated.py)
CHAIN = 64                # additions in a row's sums: at most 32 in a lane (wide rows: 8 + C / 8192), 6 over lanes, 16 over wavefronts
LAYER, RMS = 0, 1
NONE = 2


def norm_fwd(x, kind, gamma, beta, eps):
    """y, mean, rstd in 64 bits and the bounds on their errors."""
    x, g = x.double(), gamma.double() if gamma is not None else torch.ones(x.shape[1], dtype=torch.float64, device=x.device)
    b = beta.double() if beta is not None else torch.zeros_like(g)
    e = CHAIN * U
    mean = x.mean(dim=1, keepdim=True) if kind == LAYER else x.new_zeros(x.shape[0], 1)
    d = x - mean
    rstd = 1.0 / torch.sqrt((d * d).mean(dim=1, keepdim=True) + eps)
    n = d * rstd
    y = n * g + b
    em = (e + U) * x.abs().mean(dim=1, keepdim=True) if kind == LAYER else torch.zeros_like(mean)   # of the mean
    ed = em + U * d.abs()
    # squares of deviations from a mean that is off by em: their mean is off by em^2 beside the sum's own error; eps as fp32; root, quotient
    er = 0.5 * (e + 6 * U + (em * rstd) ** 2 + 2 * em * rstd * U) + 4 * U                            # of rstd, relative
    ty = g.abs() * (rstd * ed + n.abs() * (er + 2 * U)) + U * (n * g).abs() + U * y.abs() + BF16 * y.abs() + TINY
    return (y, mean[:, 0], rstd[:, 0]), (ty, em[:, 0] + U * mean[:, 0].abs() + TINY, (er * rstd)[:, 0])


def norm_bwd(dy, x, kind, gamma, mean, rstd, residual):
    """dx, dgamma, dbeta in 64 bits from the given fp32 statistics, and the bounds."""
    M, C = x.shape
    dy, x, r = dy.double(), x.double(), rstd.double()[:, None]
    g = gamma.double() if gamma is not None else torch.ones(C, dtype=torch.float64, device=x.device)
    n = (x - mean.double()[:, None] if kind == LAYER else x) * r
    t = dy * g
    s0 = t.mean(dim=1, keepdim=True) if kind == LAYER else torch.zeros_like(r)
    s1 = (t * n).mean(dim=1, keepdim=True)
    res = residual.double() if residual is not None else torch.zeros_like(x)
    dx = r * (t - s0 - n * s1)
    e = CHAIN * U
    inner = 4 * U * t.abs() + (e + 4 * U) * t.abs().mean(dim=1, keepdim=True) * (kind == LAYER) + 4 * U * s0.abs()
    inner = inner + n.abs() * ((e + 6 * U) * (t * n).abs().mean(dim=1, keepdim=True) + 8 * U * s1.abs())
    tx = r * inner + 2 * U * dx.abs() + U * (dx + res).abs() + BF16 * (dx + res).abs() + TINY
    chain = M / 64 + 48 + 4   # rows of a wavefront, teams of a workgroup, partial sums; and the products' own roundings
    return (dx + res, (dy * n).sum(0), dy.sum(0)), (tx, chain * U * (dy * n).abs().sum(0) + TINY, chain * U * dy.abs().sum(0) + TINY)


def act(name, z):
    """a(z) and a'(z) by the logistic function, which keeps its bits where 1 + tanh would cancel (z below -6)."""
    if name == NONE:
        return z, torch.ones_like(z)
    w, slope = (z, torch.ones_like(z)) if name == gated_ref.SILU else (2 * gated_ref.C * (z + gated_ref.K3 * z ** 3), 2 * gated_ref.C * (1 + 3 * gated_ref.K3 * z * z))
    q, rest = torch.sigmoid(w), torch.sigmoid(-w)
    return z * q, q + torch.where(q * rest == 0, torch.zeros_like(z), z * q * rest * slope)


def dense_fwd(x, w, nk, bias, name, residual):
    """z and y in 64 bits and the bounds."""
    s, es = gated_ref.product(x, w, nk)
    z = s + bias.double() if bias is not None else s
    ez = es + U * z.abs()
    a, _ = act(name, z)
    y = a + residual.double() if residual is not None else a
    arith = ARITH * (1 + z.abs()) * a.abs() if name != NONE else 0.0
    ey = 1.2 * ez + arith + U * y.abs()
    return (z, y), (ez + BF16 * z.abs() + TINY, ey + BF16 * y.abs() + TINY)


def dense_bwd(dh, eh, z, name):
    """dz, h and db in 64 bits from dH that is off by up to eh, and the bounds."""
    a, slope = act(name, z.double()) if z is not None else act(NONE, torch.zeros_like(dh))
    dz = dh * slope
    gate = 0.0 if name == NONE else ARITH * (1 + (z.double().abs() if z is not None else 0))
    ez = 1.2 * eh + gate * dh.abs() + 2 * U * dz.abs()
    # a column's sum: up to 256 rows of a tile, then tiles of 16 rows or more by sixteen and sixteen sums of them
    chain = min(dh.shape[0], 256) + dh.shape[0] / 256 + 20
    eb = ez.sum(0) + chain * U * (dz.abs() + ez).sum(0) + TINY
    return (dz, a, dz.sum(0)), (ez + BF16 * dz.abs() + TINY, (gate + BF16) * a.abs() + TINY, eb)


# ---- AdamW: every fp32 operation of the states written out, so that their bits are known ----
def philox(ctr, key):
    """Philox4x32-10 over uint64 arrays that hold 32-bit words."""
    c0, c1, c2, c3 = (np.asarray(c, dtype=np.uint64) for c in ctr)
    k0, k1 = key
    mask = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        p0, p1 = np.uint64(0xD2511F53) * c0, np.uint64(0xCD9E8D57) * c2
        c0, c1, c2, c3 = (p1 >> np.uint64(32)) ^ c1 ^ np.uint64(k0), p1 & mask, (p0 >> np.uint64(32)) ^ c3 ^ np.uint64(k1), p0 & mask
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return c0, c1, c2, c3


def state_bits(rows, cols, seed, step):
    """16 random bits an element: for m, for r."""
    groups = -(-cols // 4)
    row, group = np.meshgrid(np.arange(rows), np.arange(groups), indexing="ij")
    words = philox((group, row, np.full_like(row, step & 0xFFFFFFFF), np.full_like(row, (step >> 32) ^ 0x47414457)), (seed & 0xFFFFFFFF, seed >> 32))
    words = np.stack(words, axis=2).reshape(rows, -1)[:, :cols]
    return (words & np.uint64(0xFFFF)).astype(np.int64), (words >> np.uint64(16)).astype(np.int64)


E4M3 = np.array([(m / 512.0 if e == 0 else (8 + m) * 2.0 ** (e - 10)) for e in range(16) for m in range(8)][:127])   # by code


def encode_state(v, bits, root):
    """float32 v [rows x cols] -> codes, scales.  Between neighbours a and b a value at place f from a goes to b where the bits, as a number in steps of 2^-16 that
    begins at 2^-17, reach 1 - f."""
    rows, cols = v.shape
    nb = -(-cols // 32)
    codes, scales = np.zeros((rows, cols), dtype=np.uint8), np.zeros((rows, nb), dtype=np.uint8)
    for b in range(nb):
        part = v[:, 32 * b:32 * b + 32].astype(np.float64)
        top = np.abs(part).max(axis=1)
        bad = ~np.isfinite(part).all(axis=1)
        with np.errstate(divide="ignore", invalid="ignore"):
            e = np.where(bad | (top == 0), 0, np.ceil(np.log2(np.where(bad | (top == 0), 1.0, top) / 448.0) - 1e-9)).astype(int)
        for _ in range(2):   # log2 may miss by one
            e = np.where(~bad & (top > 448.0 * 2.0 ** e), e + 1, e)
            e = np.where(~bad & (top > 0) & (top <= 448.0 * 2.0 ** (e - 1.0)), e - 1, e)
        e = np.where(top == 0, 0, np.clip(e, -117, 119))
        scales[:, b] = np.where(bad, 255, e + 127)
        t = np.minimum(np.abs(np.where(bad[:, None], 0.0, part)) / 2.0 ** e[:, None], 448.0)
        t = np.where(t < 2.0 ** -6, (t.astype(np.float32) + np.float32(2.0 ** -6)).astype(np.float64) - 2.0 ** -6, t)   # its spacing there
        lo = np.clip(np.searchsorted(E4M3, t, side="right") - 1, 0, 126)
        hi = np.minimum(lo + 1, 126)
        gap = np.where(hi > lo, E4M3[hi] - E4M3[lo], 1.0)
        f = (t - E4M3[lo]) / gap
        up = f + (bits[:, 32 * b:32 * b + 32] + 0.5) / 65536.0 >= 1.0
        c = np.where(up, hi, lo)
        if root:
            c = np.where((c == 0) & (part > 0), 1, c)
        else:
            c = c | np.where(np.signbit(part), 128, 0)
        codes[:, 32 * b:32 * b + 32] = np.where(bad[:, None], 127, c)
    return codes, scales


def decode_state(codes, scales):
    v = np.concatenate([E4M3, [np.nan], -E4M3, [np.nan]])[codes]
    x = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return v * np.repeat(x, 32, axis=1)[:, :codes.shape[1]]


def adamw(p, g, m, v, root, lr, step, beta1, beta2, eps, decay, scale):
    """float32 arrays; v holds the root where `root`.  m', v' (or r') to the bit; p' in 64 bits with its bound."""
    f = np.float32
    with np.errstate(all="ignore"):
        g = (g.astype(f) * f(scale)).astype(f)
        v = (v * v).astype(f) if root else v
        m1 = (f(beta1) * m).astype(f) + (f(1.0 - beta1) * g).astype(f)
        v1 = (f(beta2) * v).astype(f) + (f(1.0 - beta2) * (g * g).astype(f)).astype(f)
        r1 = np.sqrt(v1)
        c1, c2 = 1.0 - beta1 ** step, 1.0 - beta2 ** step
        move = lr / c1 * m1.astype(np.float64) / (r1.astype(np.float64) / np.sqrt(c2) + eps)
        kept = p.astype(np.float64) * (1.0 - lr * decay)
    return m1, (r1 if root else v1), kept - move, 4 * U * np.abs(kept) + 12 * U * np.abs(move) + TINY
