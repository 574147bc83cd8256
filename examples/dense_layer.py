"""A feed-forward layer of a decoder with its norm, x + gelu(norm(x) W1 + b1) W2 + b2, trained with sampled weights by AdamW with clipping, the states of the
weights in 8 bits; then a single token through the trained layer.

    python examples/dense_layer.py [--tokens 4096 --width 768 --block 2048 --steps 20]

One step: both weights are sampled (W + R * scale, paper Eq. 3); norm, first product with bias and GELU (Z kept), second product with bias and the residual; backward dZ
and H from dY in one kernel with the first bias's gradient, the weight gradients with dL/db_t from their epilogues, the input gradient through the norm with the
gradient that comes past it; the norm of all gradients, and the update, which also writes the BF16 weights that the next step samples.  The host waits for nothing.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2505_11170_amd as gws  # noqa: E402

DEV, FMT = "cuda:0", gws.FMT_FP8_E4M3


def bf16(rows, cols):
    return torch.zeros(rows, cols, dtype=torch.bfloat16, device=DEV)


def fp32(n):
    return torch.zeros(n, device=DEV)


def eight_bits(rows, cols):
    return gws.Act8(torch.zeros(rows, cols, dtype=torch.uint8, device=DEV), torch.zeros(rows, cols // 32, dtype=torch.uint8, device=DEV))


class DenseLayer:
    """Weights stored [out x in] (w_is_nk), and the buffers that a step fills: allocated once, as they do not move between steps."""

    def __init__(self, tokens, width, block, seed=0, decay=0.01):
        if tokens % 64 or width % 256 or block % 256:
            raise ValueError(f"the weight gradients take a multiple of 64 tokens and widths of multiples of 256, not {tokens} tokens, {width} -> {block}")
        gen = torch.Generator(device=DEV).manual_seed(seed)
        self.M, self.C, self.F = tokens, width, block
        self.desc, self.vectors, self.grads, parameters = {}, {}, {}, []
        for i, (name, rows, cols) in enumerate((("up", block, width), ("down", width, block))):
            w = torch.randn(rows, cols, generator=gen, device=DEV) * cols ** -0.5
            blocks = (rows // 32, cols // 32)
            d = gws.TensorDesc(rows=rows, cols=cols, seed=gws.gws_derive_seed(seed, i), w=w.bfloat16(), w_hat=bf16(rows, cols), dw=bf16(rows, cols),
                               bt=torch.full(blocks, 6.0, device=DEV), scale=torch.zeros(blocks, device=DEV), dbt=torch.zeros(blocks, device=DEV))
            self.desc[name] = d
            parameters.append(gws.AdamWTensor(p=w, g=d.dw, m=eight_bits(rows, cols), v=eight_bits(rows, cols), w=d.w, weight_decay=decay,
                                              seed=gws.gws_derive_seed(seed, 100 + i)))
        for name, n, start in (("gamma", width, 1.0), ("beta", width, 0.0), ("b_up", block, 0.0), ("b_down", width, 0.0)):
            self.vectors[name], self.grads[name] = torch.full((n,), start, device=DEV), fp32(n)
            parameters.append(gws.AdamWTensor(p=self.vectors[name], g=self.grads[name], m=fp32(n), v=fp32(n)))
        self.parameters = gws.pack_adamw(parameters)
        M, C, F = tokens, width, block
        self.n, self.dn, self.y, self.dx, self.z, self.h, self.dz = bf16(M, C), bf16(M, C), bf16(M, C), bf16(M, C), bf16(M, F), bf16(M, F), bf16(M, F)
        self.mean, self.rstd, self.clip = fp32(M), fp32(M), fp32(2)
        need = max(gws.gws_norm_bwd_workspace_bytes(M, C), gws.gws_dense_bwd_workspace_bytes(M, F), gws.gws_dense_bwd_workspace_bytes(M, C),
                   gws.gws_grad_norm_workspace_bytes(self.parameters))
        self.workspace = torch.empty(need, dtype=torch.uint8, device=DEV)

    def sample(self, step):
        gws.gws_sample_fwd(list(self.desc.values()), FMT, step)

    def forward(self, x):
        v, d = self.vectors, self.desc
        gws.gws_norm_fwd(x, self.n, gamma=v["gamma"], beta=v["beta"], mean=self.mean, rstd=self.rstd)
        gws.gws_dense_fwd(self.n, d["up"].w_hat, self.h, bias=v["b_up"], act=gws.ACT_GELU_TANH, z=self.z, w_is_nk=True)
        gws.gws_dense_fwd(self.h, d["down"].w_hat, self.y, bias=v["b_down"], residual=x, w_is_nk=True)
        return self.y

    def backward(self, x, dy, step):
        v, g, d, ws = self.vectors, self.grads, self.desc, self.workspace
        gws.gws_dense_bwd_h(dy, None, None, dbias=g["b_down"], workspace=ws)
        gws.gws_dense_bwd(dy, d["down"].w_hat, self.z, self.dz, gws.ACT_GELU_TANH, h=self.h, dbias=g["b_up"], workspace=ws, w_is_nk=True)
        gws.gws_linear_bwd_w(self.h, dy, d["down"], step, w_is_nk=True)
        gws.gws_linear_bwd_w(self.n, self.dz, d["up"], step, w_is_nk=True)
        gws.gws_gemm_bf16(self.dz, d["up"].w_hat, self.dn)                  # dn = dZ W: the weight the other way round
        gws.gws_norm_bwd(self.dn, x, self.dx, self.rstd, mean=self.mean, gamma=v["gamma"], residual=dy, dgamma=g["gamma"], dbeta=g["beta"], workspace=ws)
        return self.dx

    def update(self, step, rate, limit=1.0):
        gws.gws_grad_norm(self.parameters, self.clip, self.workspace, max_norm=limit)
        gws.gws_adamw(self.parameters, lr=rate, step=step, grad_scale=self.clip[1:])

    def token(self, x):
        """Serving: x [1 x width] through the weights as they were last sampled; nothing is kept."""
        v, d, n, h, y = self.vectors, self.desc, bf16(1, self.C), bf16(1, self.F), bf16(1, self.C)
        gws.gws_norm_fwd(x, n, gamma=v["gamma"], beta=v["beta"])
        gws.gws_dense_fwd(n, d["up"].w_hat, h, bias=v["b_up"], act=gws.ACT_GELU_TANH, w_is_nk=True)
        gws.gws_dense_fwd(h, d["down"].w_hat, y, bias=v["b_down"], residual=x, w_is_nk=True)
        return y


def train(tokens, width, block, steps, rate=1e-3, say=print):
    """Losses of the steps, the layer and its input: it learns to reproduce another layer of its kind."""
    teacher, layer = DenseLayer(tokens, width, block, seed=1), DenseLayer(tokens, width, block, seed=2)
    teacher.sample(0)
    gen = torch.Generator(device=DEV).manual_seed(3)
    x = torch.randn(tokens, width, generator=gen, device=DEV).bfloat16()
    goal = teacher.forward(x).float().clone()
    losses = []
    for step in range(1, steps + 1):
        layer.sample(step)
        error = layer.forward(x).float() - goal
        losses.append((error ** 2).mean() / (goal ** 2).mean())
        dy = (error * (2.0 / tokens)).bfloat16()              # of the loss summed over columns, averaged over tokens
        layer.backward(x, dy, step)
        layer.update(step, rate)
    for step in range(0, steps, max(1, steps // 10)):
        say(f"step {step + 1}: relative error {float(losses[step]):.4f}")
    say(f"last gradient norm {float(layer.clip[0]):.3f}, factor {float(layer.clip[1]):.3f}")
    return [float(v) for v in losses], layer, x


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--width", type=int, default=768)
    ap.add_argument("--block", type=int, default=2048)
    ap.add_argument("--steps", type=int, default=20)
    a = ap.parse_args()
    _, layer, x = train(a.tokens, a.width, a.block, a.steps)
    n = 2 * a.width * a.block
    print(f"states of the weights: {2 * n * (8 + 8 / 32) / 8 / 2**20:.1f} MiB, in 32 bits {2 * n * 4 / 2**20:.1f}")
    print("one token:", layer.token(x[:1])[0, :4].tolist())


if __name__ == "__main__":
    main()
