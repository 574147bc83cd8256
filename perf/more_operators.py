"""What a decoder layer needs around its sampled products in training and serving, and the update at the end of a step, as measurable
cases.

Six operators.  M tokens; o is the product by elements, * between matrices the matrix product; sums over a row are over its C columns:

 ``norm_fwd``   Y = (X - mean) rstd o gamma + beta with mean and rstd = 1 / sqrt(variance + eps) of each row, kept for the backward
                pass; root mean square form ("rms"): Y = X rstd o gamma, rstd = 1 / sqrt(mean of squares + eps).
 ``norm_bwd``   with n = (X - mean) rstd and t = dY o gamma: dX = rstd (t - mean(t) - n mean(t n)) + R, where R is the gradient that
                comes past the norm; dgamma = sum over tokens of dY o n, dbeta = sum of dY ("rms": no mean(t), n = X rstd).
 ``dense_fwd``  Z = X * W + b, Y = a(Z) + R; a is SiLU, GELU in its tanh form, or nothing; Z kept for the backward pass, R a residual.
 ``dense_bwd``  from the gradient of the product that follows (dH = dY * Wd^T, ``from`` "dy") or from dH ("dh"), and the kept Z:
                dZ = dH o a'(Z), H = a(Z) again for that product's weight gradient, db = sum over tokens of dZ.
 ``adamw``      over a list of tensors, step t: m = b1 m + (1 - b1) g, v = b2 v + (1 - b2) g^2,
                p = p (1 - lr decay) - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps), and the BF16 copy w of p.  With ``clip``
                the gradients are first multiplied by min(1, limit / norm of all of them).  The states m and v are held in 32 bits,
                or those of the matrices in 8: m and r = sqrt(v) as E4M3 values, 32 neighbouring ones of a row sharing a power of two
                X, the smallest for which the largest of them is at most 448 X; rounded up or down at random, so that a mean over
                many steps moves however small a step's share of it is; r > 0 never becomes 0.

The random bits of that rounding are those of the counter-based generator Philox4x32-10, of which seed, step, row and column are the
input: key = seed, counter = (column / 4, row, step mod 2^32, step / 2^32 xor 0x47414457); column 4 q + e has word e, its low half for m and its
high half for r.

``exact`` computes the same outputs in 64 bits and shares no code with the plain form.
"""
import math

import torch

own = False

DEV = "cuda:0"
BLOCK = 32
GELU_C, GELU_K = math.sqrt(2.0 / math.pi), 0.044715
EPS = 1e-5                                # of the norms
LR, BETA1, BETA2, ADAM_EPS, DECAY, LIMIT = 3e-4, 0.9, 0.95, 1e-8, 0.1, 1.0
MAX_FLOPS = 2 * 8192 * 2048 * 5632        # of the largest listed product
MAX_ELEMENTS = 8192 * 5632                # of the largest drawn norm
MAX_PARAMETERS = 4 * (4 * 2048 * 2048 + 2 * 2048 * 5632)


# ---------------------------------------------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------------------------------------------
def _norm(way, M, C, *, kind="layer", extra=True):
    """extra: forward, mean and rstd are kept; backward, a gradient comes past the norm."""
    return {"op": "norm_" + way, "M": M, "C": C, "kind": kind, "extra": extra}


def _dense_fwd(M, K, N, *, nk, act="gelu", residual=False, keep=False):
    return {"op": "dense_fwd", "M": M, "K": K, "N": N, "nk": nk, "act": act, "residual": residual, "keep": keep}


def _dense_bwd(M, D, F, *, nk, act="gelu", src="dy"):
    return {"op": "dense_bwd", "M": M, "K": D, "N": F, "nk": nk, "act": act, "from": src}


def _adamw(width, block, layers, *, bits, clip, matrices=True):
    return {"op": "adamw", "width": width, "block": block, "layers": layers, "bits": bits, "clip": clip, "matrices": matrices}


def listed():
    return [
        # serving: the norm in front of one token's products in the 1B decoder; nothing is kept
        dict(_norm("fwd", 1, 2048, kind="rms", extra=False), name="norm_fwd_1_token"),
        # training: a micro-batch
        dict(_norm("fwd", 8192, 2048), name="norm_fwd_8192x2048"),
        # a short, uneven batch at the 124M model's width, with the gradient that comes past the norm
        dict(_norm("bwd", 1021, 768), name="norm_bwd_1021x768"),
        dict(_norm("bwd", 8192, 2048), name="norm_bwd_8192x2048"),
        # serving: one token through a feed-forward layer's first weight
        dict(_dense_fwd(1, 2048, 5632, nk=True), name="dense_fwd_1_token"),
        # the layer's second product for an uneven batch: bias and the residual stream, weights stored [K x N]
        dict(_dense_fwd(1021, 2048, 768, nk=False, act="none", residual=True), name="dense_fwd_ragged_residual"),
        # its first product for a training micro-batch, Z kept
        dict(_dense_fwd(8192, 2048, 5632, nk=True, keep=True), name="dense_fwd_8192_keep"),
        # the backward pass of both batches through the second product
        dict(_dense_bwd(1021, 768, 2048, nk=False), name="dense_bwd_ragged"),
        dict(_dense_bwd(8192, 2048, 5632, nk=True), name="dense_bwd_8192"),
        # biases and norms of twelve layers alone, as where the matrices are frozen
        dict(_adamw(768, 2048, 12, bits=32, clip=True, matrices=False), name="adamw_vectors"),
        # twelve layers of the 124M model's width, clipped
        dict(_adamw(768, 2048, 12, bits=32, clip=True), name="adamw_12_layers_32_bit"),
        # four layers of the 1B decoder's width, states of the matrices in 8 bits
        dict(_adamw(2048, 5632, 4, bits=8, clip=False), name="adamw_4_layers_8_bit"),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _width(rng, low, high, step=32):
    return max(low, min(high, step * int(round(math.exp(rng.uniform(math.log(low), math.log(high))) / step))))


def draw(rng):
    op = rng.choice(["norm_fwd", "norm_bwd", "dense_fwd", "dense_fwd", "dense_bwd", "adamw"])
    if op in ("norm_fwd", "norm_bwd"):
        C = _log(rng, 64, 8192)
        return _norm(op[5:], _log(rng, 1, min(16384, MAX_ELEMENTS // C)), C, kind=rng.choice(["layer", "rms"]), extra=rng.random() < 0.7)
    if op == "adamw":
        width, block, bits, clip = _log(rng, 100, 2048), _log(rng, 200, 5632), rng.choice([32, 8]), rng.random() < 0.5
        one = 4 * width * width + 2 * width * block
        layers = _log(rng, 1, max(1, min(24, MAX_PARAMETERS // (one * (1 if bits == 8 else 2)))))
        return _adamw(width, block, layers, bits=bits, clip=clip, matrices=rng.random() < 0.85)
    K, N = _width(rng, 256, 5632), _width(rng, 256, 5632)
    M = _log(rng, 1, min(8192, MAX_FLOPS // (2 * K * N)))
    nk, act = rng.random() < 0.5, rng.choice(["gelu", "silu", "none"])
    if op == "dense_fwd":
        return _dense_fwd(M, K, N, nk=nk, act=act, residual=rng.random() < 0.5, keep=rng.random() < 0.5)
    return _dense_bwd(M, K, N, nk=nk, act=rng.choice(["gelu", "silu"]), src=rng.choice(["dy", "dy", "dh"]))


# ---------------------------------------------------------------------------------------------------------------
# The plain form
# ---------------------------------------------------------------------------------------------------------------
def _gate(act, z):
    """a(z) and a'(z): with q the logistic function of w(z), a = z q and a' = q + z q (1 - q) w'(z)."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "silu":
        q = 1.0 / (1.0 + torch.exp(-z))
        return z * q, q * (1.0 + z * (1.0 - q))
    z2 = z * z
    q = 1.0 / (1.0 + torch.exp(-2.0 * GELU_C * z * (1.0 + GELU_K * z2)))
    return z * q, q + z * q * (1.0 - q) * (2.0 * GELU_C * (1.0 + 3.0 * GELU_K * z2))


def _mul32(a, b):
    """High and low halves of the product of 32-bit numbers held in int64."""
    a1, a0 = a >> 16, a & 0xFFFF
    low, high = a0 * b, a1 * b
    whole = (high << 16) + low            # mod 2^64
    return (high + (low >> 16)) >> 16, whole & 0xFFFFFFFF


def _philox(rows, groups, step, seed):
    """Four words for every group of every row, int64 [rows, groups] each."""
    c0 = torch.arange(groups, device=DEV).expand(rows, groups)
    c1 = torch.arange(rows, device=DEV)[:, None].expand(rows, groups)
    c2, c3 = torch.full_like(c0, step & 0xFFFFFFFF), torch.full_like(c0, (step >> 32) ^ 0x47414457)
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        h0, l0 = _mul32(c0, 0xD2511F53)
        h1, l1 = _mul32(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return torch.stack([c0, c1, c2, c3], dim=2)


def _random_codes(v, bits16, never_zero):
    """[rows x cols] in 32 bits -> E4M3 values and E8M0 scales, rounded at random with 16 bits an element."""
    rows, cols = v.shape
    nb = -(-cols // BLOCK)
    pad = lambda t: torch.cat([t, t.new_zeros(rows, nb * BLOCK - cols)], dim=1).reshape(rows, nb, BLOCK)  # noqa: E731
    b = pad(v)
    top = b.abs().amax(dim=2).view(torch.int32)
    biased = ((top >> 23) - 8 + ((top & 0x7FFFFF) > 0x600000)).clamp(min=10)     # 1.75 2^8 = 448
    biased = torch.where(top == 0, torch.full_like(biased, 127), biased)
    t = b.abs() * ((254 - biased) << 23).view(torch.float32)[:, :, None]
    small = t < 2.0 ** -6
    raw = torch.where(small, t + 2.0 ** -6, t).view(torch.int32) + (pad(bits16.to(torch.int32)) << 4) + 8
    code = (raw >> 20) - torch.where(small, 968, 960)
    if never_zero:
        code = torch.where((code == 0) & (b > 0), torch.ones_like(code), code)
    code = code | ((b < 0).to(torch.int32) << 7)
    return code.reshape(rows, nb * BLOCK)[:, :cols].to(torch.uint8).view(torch.float8_e4m3fn), biased.to(torch.uint8).view(torch.float8_e8m0fnu)


def _values(codes, scales):
    x = (scales.view(torch.uint8).to(torch.int32) << 23).view(torch.float32)
    return codes.to(torch.float32) * x.repeat_interleave(BLOCK, dim=1)[:, :codes.shape[1]]


def _put(to, v):
    """In place, as the framework's call updates the user's buffers."""
    if to.dtype.itemsize == 1:
        to.view(torch.uint8).copy_(v.view(torch.uint8))
    else:
        to.copy_(v)


def _plain_adamw(s):
    scale = 1.0
    if s["clip"]:
        total = torch.zeros((), dtype=torch.float64, device=DEV)
        for t in s["tensors"]:
            total = total + (t["g"].double() ** 2).sum()
        norm = total.sqrt()
        s["clipped"][0] = norm
        s["clipped"][1] = torch.where(norm > LIMIT, LIMIT / norm, torch.ones_like(norm))
        scale = s["clipped"][1]
    c1, c2 = 1.0 - BETA1 ** s["step"], 1.0 - BETA2 ** s["step"]
    for t in s["tensors"]:
        p, g = t["p"], t["g"].float() * scale
        m, v = (_values(t["m"], t["m_scale"]), _values(t["v"], t["v_scale"])) if "m_scale" in t else (t["m"], t["v"])
        if "m_scale" in t:
            v = v * v
        m = m * BETA1 + g * (1.0 - BETA1)
        v = v * BETA2 + (g * g) * (1.0 - BETA2)
        r = v.sqrt()
        p = p * (1.0 - LR * t["decay"]) - (LR / c1) * m / (r * (1.0 / math.sqrt(c2)) + ADAM_EPS)
        _put(t["p"], p)
        _put(t["w"], p.bfloat16())
        if "m_scale" in t:
            rows, cols = p.shape
            words = _philox(rows, -(-cols // 4), s["step"], t["seed"]).reshape(rows, -1)[:, :cols]
            for k, x, half in (("m", m, words & 0xFFFF), ("v", r, words >> 16)):
                codes, scales = _random_codes(x, half, never_zero=k == "v")
                _put(t[k], codes)
                _put(t[k + "_scale"], scales)
        else:
            _put(t["m"], m)
            _put(t["v"], v)
    return _adamw_outputs(s)


def _plain(s):
    op = s["op"]
    if op == "adamw":
        return _plain_adamw(s)
    if op == "norm_fwd":
        x = s["x"].float()
        mean = x.mean(dim=1) if s["kind"] == "layer" else torch.zeros(x.shape[0], device=DEV)
        d = x - mean[:, None]
        rstd = 1.0 / torch.sqrt((d * d).mean(dim=1) + EPS)
        y = d * rstd[:, None] * s["gamma"]
        if s["kind"] == "layer":
            y = y + s["beta"]
        out = {"y": y.bfloat16()}
        if s["extra"]:
            out["rstd"] = rstd
            if s["kind"] == "layer":
                out["mean"] = mean
        return out
    if op == "norm_bwd":
        x, dy, rstd = s["x"].float(), s["dy"].float(), s["rstd"][:, None]
        n = (x - s["mean"][:, None] if s["kind"] == "layer" else x) * rstd
        t = dy * s["gamma"]
        dx = t - n * (t * n).mean(dim=1, keepdim=True)
        if s["kind"] == "layer":
            dx = dx - t.mean(dim=1, keepdim=True)
        dx = dx * rstd
        if s["extra"]:
            dx = dx + s["r"].float()
        out = {"dx": dx.bfloat16(), "dgamma": (dy * n).sum(dim=0)}
        if s["kind"] == "layer":
            out["dbeta"] = dy.sum(dim=0)
        return out
    if op == "dense_fwd":
        w = s["w"].float()
        z = s["x"].float() @ (w.t() if s["nk"] else w) + s["b"]
        y = _gate(s["act"], z)[0]
        if s["residual"]:
            y = y + s["r"].float()
        out = {"y": y.bfloat16()}
        if s["keep"]:
            out["z"] = z.bfloat16()
        return out
    if s["from"] == "dy":
        w = s["wd"].float()
        dh = s["dy"].float() @ (w if s["nk"] else w.t())
    else:
        dh = s["dh"].float()
    a, slope = _gate(s["act"], s["z"].float())
    dz = dh * slope
    return {"dz": dz.bfloat16(), "h": a.bfloat16(), "db": dz.sum(dim=0)}


# ---------------------------------------------------------------------------------------------------------------
# The framework's calls
# ---------------------------------------------------------------------------------------------------------------
def _own(s):
    import paper_2505_11170_amd as gws

    op = s["op"]
    if op == "adamw":
        if s["clip"]:
            gws.gws_grad_norm(s["packed"], s["clipped"], s["workspace"], max_norm=LIMIT)
        gws.gws_adamw(s["packed"], lr=LR, step=s["step"], beta1=BETA1, beta2=BETA2, eps=ADAM_EPS, grad_scale=s["clipped"][1:] if s["clip"] else None)
        return _adamw_outputs(s)
    if op in ("norm_fwd", "norm_bwd"):
        kind = gws.NORM_LAYER if s["kind"] == "layer" else gws.NORM_RMS
        if op == "norm_fwd":
            gws.gws_norm_fwd(s["x"], s["y"], kind, gamma=s["gamma"], beta=s.get("beta"), eps=EPS, mean=s.get("mean"), rstd=s.get("rstd"))
            return {k: s[k] for k in ("y", "rstd", "mean") if k in s}
        gws.gws_norm_bwd(s["dy"], s["x"], s["dx"], s["rstd"], kind, mean=s.get("mean"), gamma=s["gamma"], residual=s.get("r"), dgamma=s["dgamma"],
                         dbeta=s.get("dbeta"), workspace=s["workspace"])
        return {k: s[k] for k in ("dx", "dgamma", "dbeta") if k in s}
    act = {"none": gws.ACT_NONE, "silu": gws.ACT_SILU, "gelu": gws.ACT_GELU_TANH}[s["act"]]
    if op == "dense_fwd":
        gws.gws_dense_fwd(s["x"], s["w"], s["y"], bias=s["b"], act=act, residual=s.get("r"), z=s.get("z"), w_is_nk=s["nk"])
        return {k: s[k] for k in ("y", "z") if k in s}
    if s["from"] == "dy":
        gws.gws_dense_bwd(s["dy"], s["wd"], s["z"], s["dz"], act, h=s["h"], dbias=s["db"], workspace=s["workspace"], w_is_nk=s["nk"])
    else:
        gws.gws_dense_bwd_h(s["dh"], s["z"], s["dz"], act, h=s["h"], dbias=s["db"], workspace=s["workspace"])
    return {k: s[k] for k in ("dz", "h", "db")}


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------------------------
def _buffer(rows, cols, dtype=torch.bfloat16):
    """Zeros, in rows of a whole number of eights, as the framework takes them."""
    return torch.zeros(rows, -(-cols // 8) * 8, device=DEV, dtype=dtype)[:, :cols]


def _normal(gen, rows, cols, std, dtype=torch.bfloat16):
    v = _buffer(rows, cols, dtype)
    v.copy_(torch.randn(rows, cols, generator=gen, device=DEV).mul_(std))
    return v


def _activations(gen, rows, cols):
    """As a layer meets them: channels of different sizes and offsets, a few of them large, and now and then a padding token of zeros."""
    v = torch.randn(rows, cols, generator=gen, device=DEV) + 0.3 * torch.randn(1, cols, generator=gen, device=DEV) + 0.2
    v *= torch.exp(0.5 * torch.randn(1, cols, generator=gen, device=DEV))
    v *= 1.0 + 15.0 * (torch.rand(1, cols, generator=gen, device=DEV) < 0.01)
    out = _buffer(rows, cols)
    out.copy_(v * (torch.rand(rows, 1, generator=gen, device=DEV) >= 0.02))
    return out


def _vector(gen, n, mean, std):
    return mean + std * torch.randn(n, generator=gen, device=DEV)


def _shapes(c):
    """Matrices [out x in] and vectors of the layers: q, k and v together, the projection behind them, and the two of the feed-forward layer."""
    w, f = c["width"], c["block"]
    matrices = [(3 * w, w), (w, w), (f, w), (w, f)] if c["matrices"] else []
    return [s for _ in range(c["layers"]) for s in matrices + [(n,) for n in (3 * w, w, f, w, w, w, w, w)]]


class _Flat:
    """Matrices side by side in one buffer, as a training program holds its parameters and states, each in rows of a whole number of eights and
    from a whole cache line on."""

    def __init__(self, shapes, dtype, step=8):
        self.places, n = [], 0
        for shape in shapes:
            rows, cols = shape if len(shape) == 2 else (1, shape[0])
            ld = -(-cols // step) * step
            self.places.append((n, rows, ld, cols, len(shape)))
            n += -(-rows * ld // 128) * 128
        self.all = torch.zeros(n, device=DEV, dtype=dtype)

    def __getitem__(self, i):
        at, rows, ld, cols, dims = self.places[i]
        v = self.all[at:at + rows * ld].view(rows, ld)[:, :cols]
        return v if dims == 2 else v[0]


def _prepare_adamw(s, gen):
    """Parameters, their gradients and their states some steps into a training run."""
    s["step"] = 100
    shapes = _shapes(s)
    held = [i for i, shape in enumerate(shapes) if s["bits"] == 8 and len(shape) == 2]      # in 8 bits
    wide = [i for i in range(len(shapes)) if i not in set(held)]
    s["flat"] = {"p": _Flat(shapes, torch.float32), "w": _Flat(shapes, torch.bfloat16)}
    for k in ("m", "v"):
        s["flat"][k] = _Flat([shapes[i] for i in wide], torch.float32)
        if held:
            s["flat"][k + "8"] = _Flat([shapes[i] for i in held], torch.uint8)
            s["flat"][k + "8_scale"] = _Flat([(shapes[i][0], -(-shapes[i][1] // BLOCK)) for i in held], torch.uint8, step=1)
    s["tensors"] = []
    for i, shape in enumerate(shapes):
        matrix = len(shape) == 2
        t = {"decay": DECAY if matrix else 0.0, "seed": 0x9E3779B97F4A7C15 * (i + 1) & 0xFFFFFFFFFFFFFFFF, "p": s["flat"]["p"][i], "w": s["flat"]["w"][i]}
        rows, cols = shape if matrix else (1, shape[0])
        t["p"].copy_(_normal(gen, rows, cols, 0.02, torch.float32).reshape(shape))
        t["g"] = _normal(gen, rows, cols, 1e-3, torch.bfloat16 if matrix else torch.float32)   # vectors' gradients are sums in 32 bits
        t["g"] = t["g"] if matrix else t["g"][0]
        for k in ("m", "v"):
            if i in held:
                x = torch.randn(rows, cols, generator=gen, device=DEV).mul_(3e-4)
                if k == "v":
                    x = x.abs().mul_(3.0).add_(1e-6)      # its root
                codes, scales = _random_codes(x, torch.full(shape, 0x8000, device=DEV), never_zero=k == "v")
                t[k], t[k + "_scale"] = (s["flat"][k + name][held.index(i)].view(d) for name, d in (("8", torch.float8_e4m3fn), ("8_scale", torch.float8_e8m0fnu)))
                _put(t[k], codes)
                _put(t[k + "_scale"], scales)
            else:
                t[k] = s["flat"][k][wide.index(i)]
                x = _normal(gen, rows, cols, 3e-4 if k == "m" else 1e-3, torch.float32).reshape(shape)
                t[k].copy_(x if k == "m" else x * x + 1e-12)
        s["tensors"].append(t)
    if s["clip"]:
        s["clipped"] = torch.zeros(2, device=DEV)     # the norm, and what the gradients are multiplied by
    if own:
        import paper_2505_11170_amd as gws

        def state(t, k):
            return gws.Act8(t[k], t[k + "_scale"]) if k + "_scale" in t else t[k]

        s["packed"] = gws.pack_adamw([gws.AdamWTensor(p=t["p"], g=t["g"], m=state(t, "m"), v=state(t, "v"), w=t["w"], weight_decay=t["decay"], seed=t["seed"])
                                      for t in s["tensors"]])
        s["workspace"] = torch.empty(gws.gws_grad_norm_workspace_bytes(s["packed"]), dtype=torch.uint8, device=DEV)
    return s


def _adamw_outputs(s):
    out = {k: f.all for k, f in s["flat"].items()}
    for k in ("m8", "v8"):
        if k in out:
            out[k], out[k + "_scale"] = out[k].view(torch.float8_e4m3fn), out[k + "_scale"].view(torch.float8_e8m0fnu)
    if s["clip"]:
        out["clipped"] = s["clipped"]
    return out


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    s = dict(case)
    op = s["op"]
    if op == "adamw":
        return _prepare_adamw(s, gen)
    M = s["M"]
    workspace = lambda nbytes: torch.empty(nbytes(), dtype=torch.uint8, device=DEV) if own else None  # noqa: E731
    if own:
        import paper_2505_11170_amd as gws
    if op in ("norm_fwd", "norm_bwd"):
        C, layer = s["C"], s["kind"] == "layer"
        s["x"], s["gamma"] = _activations(gen, M, C), _vector(gen, C, 1.0, 0.1)
        if op == "norm_fwd":
            if layer:
                s["beta"] = _vector(gen, C, 0.0, 0.1)
            s["y"] = _buffer(M, C)
            for k in (("rstd", "mean") if layer else ("rstd",)) if s["extra"] else ():
                s[k] = torch.zeros(M, device=DEV)
            return s
        x = s["x"].double()                                # what the forward pass kept
        mean = x.mean(dim=1) if layer else x.new_zeros(M)
        s["rstd"] = (1.0 / torch.sqrt(((x - mean[:, None]) ** 2).mean(dim=1) + EPS)).float()
        if layer:
            s["mean"], s["dbeta"] = mean.float(), torch.zeros(C, device=DEV)
        s["dy"], s["dx"], s["dgamma"] = _normal(gen, M, C, 1e-3), _buffer(M, C), torch.zeros(C, device=DEV)
        if s["extra"]:
            s["r"] = _normal(gen, M, C, 1e-3)
        s["workspace"] = workspace(lambda: gws.gws_norm_bwd_workspace_bytes(M, C))
        return s
    K, N, nk = s["K"], s["N"], s["nk"]
    if op == "dense_fwd":
        s["x"], s["w"], s["b"] = _normal(gen, M, K, 1.0), _normal(gen, *((N, K) if nk else (K, N)), 0.02), _vector(gen, N, 0.0, 0.1)
        s["y"] = _buffer(M, N)
        if s["residual"]:
            s["r"] = _normal(gen, M, N, 1.0)
        if s["keep"]:
            s["z"] = _buffer(M, N)
        return s
    s["z"] = _normal(gen, M, N, 0.02 * math.sqrt(K))       # what the forward pass kept
    if s["from"] == "dy":
        # the product that follows, N -> K columns, its weight stored [N x K] or (nk) [K x N]
        s["dy"], s["wd"] = _normal(gen, M, K, 1e-3), _normal(gen, *((K, N) if nk else (N, K)), 0.02)
    else:
        s["dh"] = _normal(gen, M, N, 1e-3)
    s["dz"], s["h"], s["db"] = _buffer(M, N), _buffer(M, N), torch.zeros(N, device=DEV)
    s["workspace"] = workspace(lambda: gws.gws_dense_bwd_workspace_bytes(M, N))
    return s


# ---------------------------------------------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------
def work(case):
    c, op = case, case["op"]
    if op == "adamw":
        n, nbytes = 0, 0
        for shape in _shapes(c):
            k = math.prod(shape)
            n += k
            kept = 2 * (k + shape[0] * -(-shape[1] // BLOCK)) if len(shape) == 2 and c["bits"] == 8 else 8 * k
            nbytes += 8 * k + 2 * k + (2 if len(shape) == 2 else 4) * k + 2 * kept     # p in and out, w, g, states in and out
        return {"bytes": nbytes, "flops": (14 + (2 if c["clip"] else 0)) * n}
    M = c["M"]
    if op in ("norm_fwd", "norm_bwd"):
        C, vectors = c["C"], 2 if c["kind"] == "layer" else 1
        if op == "norm_fwd":
            return {"bytes": 4 * M * C + 4 * vectors * (C + (M if c["extra"] else 0)), "flops": 7 * M * C}
        return {"bytes": (8 if c["extra"] else 6) * M * C + 4 * vectors * (M + C) + 4 * C, "flops": 14 * M * C}
    K, N = c["K"], c["N"]
    if op == "dense_fwd":
        return {"bytes": 2 * M * K + 2 * K * N + 4 * N + 2 * M * N * (1 + c["residual"] + c["keep"]), "flops": 2 * M * K * N + 8 * M * N}
    source, product = (2 * M * K + 2 * K * N, 2 * M * K * N) if c["from"] == "dy" else (2 * M * N, 0)
    return {"bytes": source + 6 * M * N + 4 * N, "flops": product + 12 * M * N}


# ---------------------------------------------------------------------------------------------------------------
# The definition in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def _act64(name, z):
    if name == "none":
        return z, torch.ones_like(z)
    if name == "silu":
        a = z * torch.sigmoid(z)
        return a, torch.sigmoid(z) + a * torch.sigmoid(-z)
    t = torch.tanh(GELU_C * (z + GELU_K * z ** 3))
    return 0.5 * z * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * GELU_C * (1.0 + 3.0 * GELU_K * z * z)


def _held64(codes, scales):
    c = codes.view(torch.uint8).to(torch.int64)
    e, f = (c >> 3) & 15, (c & 7).double()
    pow2 = lambda n: ((n + 1023) << 52).view(torch.float64)  # noqa: E731
    v = torch.where(e == 0, f / 512.0, (8.0 + f) * pow2(e - 10))
    block = torch.arange(codes.shape[1], device=codes.device) // BLOCK
    return torch.where(c >= 128, -v, v) * pow2(scales.view(torch.uint8).long()[:, block] - 127)


def _exact_adamw(s):
    k, factor = s["step"], torch.ones((), dtype=torch.float64, device=DEV)
    # Rounded at random: in 64 bits the same bits round the same way but for values within their last bit of the border.
    out = {key: None if "8" in key else f.all.double() for key, f in s["flat"].items()}
    at = lambda key, t: torch.as_strided(out[key], t.shape, t.stride(), t.storage_offset())  # noqa: E731
    if s["clip"]:
        norm = torch.sqrt(sum(torch.sum(t["g"].double().square()) for t in s["tensors"]))
        factor = torch.clamp(LIMIT / norm, max=1.0)
        out["clipped"] = torch.stack([norm, factor])
    for t in s["tensors"]:
        g, held = t["g"].double() * factor, "m_scale" in t
        m = _held64(t["m"], t["m_scale"]) if held else at("m", t["m"])
        v = _held64(t["v"], t["v_scale"]).square() if held else at("v", t["v"])
        m.mul_(BETA1).add_(g, alpha=1 - BETA1)
        v.mul_(BETA2).addcmul_(g, g, value=1 - BETA2)
        step = (m / (1 - BETA1 ** k)).div_((v / (1 - BETA2 ** k)).sqrt_().add_(ADAM_EPS)).mul_(LR)
        p = at("p", t["p"])
        p.mul_(1 - LR * t["decay"]).sub_(step)
        at("w", t["w"]).copy_(p)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    op = s["op"]
    if op == "adamw":
        return _exact_adamw(s)
    d = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    if op == "norm_fwd":
        layer = s["kind"] == "layer"
        var, mean = torch.var_mean(d["x"], dim=1, correction=0)
        rstd = torch.rsqrt((var if layer else d["x"].square().mean(1)) + EPS)
        y = (d["x"] - mean[:, None] if layer else d["x"]) * torch.outer(rstd, d["gamma"])
        out = {"y": y + d["beta"] if layer else y}
        if s["extra"]:
            out["rstd"] = rstd
            if layer:
                out["mean"] = mean
        return out
    if op == "norm_bwd":
        layer, C = s["kind"] == "layer", s["C"]
        n = d["x"] * d["rstd"][:, None]
        if layer:
            n -= (d["mean"] * d["rstd"])[:, None]
        t = d["dy"] * d["gamma"]
        along = (t * n).sum(1) / C
        dx = t - n * along[:, None] - (t.sum(1) / C if layer else torch.zeros_like(along))[:, None]
        dx *= d["rstd"][:, None]
        out = {"dx": dx + d["r"] if s["extra"] else dx, "dgamma": torch.sum(n * d["dy"], 0)}
        if layer:
            out["dbeta"] = torch.sum(d["dy"], 0)
        return out
    if op == "dense_fwd":
        z = torch.addmm(d["b"], d["x"], d["w"].T.contiguous() if s["nk"] else d["w"])
        y = _act64(s["act"], z)[0]
        out = {"y": y + d["r"] if s["residual"] else y}
        if s["keep"]:
            out["z"] = z
        return out
    dh = d["dh"] if s["from"] == "dh" else torch.mm(d["dy"], d["wd"] if s["nk"] else d["wd"].T.contiguous())
    a, slope = _act64(s["act"], d["z"])
    return {"dz": slope * dh, "h": a, "db": torch.sum(slope * dh, 0)}
