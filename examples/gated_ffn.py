"""A gated feed-forward block trained with sampled weights, its activations kept in 8 bits between the passes; then single tokens
through the trained weights.

    python examples/gated_ffn.py [--tokens 8192 --width 2048 --block 5632 --steps 20]

One step: the three weights are sampled (W + R * scale, paper Eq. 3); forward H = SiLU(X Wg) * (X Wu), Y = H Wd, with X, G and U kept as
E4M3 codes; backward dG, dU and H from dY in one kernel, the input gradient, and the three weight gradients with dL/db_t from their
epilogues; then plain gradient descent on the weights.  The block learns to reproduce a random block of its own kind.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2505_11170_amd as gws  # noqa: E402

DEV, FMT = "cuda:0", gws.FMT_FP8_E4M3


def act8(rows, cols):
    return gws.Act8(torch.zeros(rows, cols, dtype=torch.uint8, device=DEV), torch.zeros(rows, cols // 32, dtype=torch.uint8, device=DEV))


def bf16(rows, cols):
    return torch.zeros(rows, cols, dtype=torch.bfloat16, device=DEV)


class GatedFFN:
    """Weights stored [out x in] (w_is_nk), and the buffers that a step fills: allocated once, as they do not move between steps."""

    def __init__(self, tokens, width, block, seed=0):
        # the weight gradients take tokens by 64 and weights by 256 x 256 (0: refused); gate and up have one shape, down its transpose
        need = gws.gws_linear_bwd_w_act8_workspace_bytes(gws.TensorDesc(rows=block, cols=width, seed=0), tokens, w_is_nk=True)
        if need == 0:
            raise ValueError(f"the weight gradients take a multiple of 64 tokens and widths of multiples of 256, not {tokens} tokens, {width} -> {block}")
        gen = torch.Generator(device=DEV).manual_seed(seed)
        self.M, self.K, self.F = tokens, width, block
        self.master, self.desc = {}, {}
        for i, (name, rows, cols) in enumerate((("gate", block, width), ("up", block, width), ("down", width, block))):
            w = torch.randn(rows, cols, generator=gen, device=DEV) * cols ** -0.5
            self.master[name] = w
            blocks = (rows // 32, cols // 32)
            self.desc[name] = gws.TensorDesc(
                rows=rows, cols=cols, seed=gws.gws_derive_seed(seed, i), w=w.bfloat16(), w_hat=bf16(rows, cols), dw=bf16(rows, cols),
                bt=torch.full(blocks, 6.0, device=DEV), scale=torch.zeros(blocks, device=DEV), dbt=torch.zeros(blocks, device=DEV))
        M, K, F = tokens, width, block
        self.x8 = act8(M, K)
        self.saved = gws.GatedSaved(g8=act8(M, F), u8=act8(M, F))
        self.h, self.y, self.dx, self.dg, self.du = bf16(M, F), bf16(M, K), bf16(M, K), bf16(M, F), bf16(M, F)
        self.workspace = torch.empty(need, dtype=torch.uint8, device=DEV)

    def sample(self, step):
        gws.gws_sample_fwd(list(self.desc.values()), FMT, step)

    def forward(self, x):
        d = self.desc
        gws.gws_act8_encode(x, self.x8)
        gws.gws_gated_fwd(x, d["gate"].w_hat, d["up"].w_hat, self.h, gws.ACT_SILU, saved=self.saved, w_is_nk=True)
        gws.gws_gemm_bf16(self.h, d["down"].w_hat, self.y, w_is_nk=True)
        return self.y

    def backward(self, dy, step):
        d = self.desc
        gws.gws_gated_bwd(dy, d["down"].w_hat, self.saved, self.dg, self.du, gws.ACT_SILU, h=self.h, w_is_nk=True)
        gws.gws_linear_bwd_w(self.h, dy, d["down"], step, w_is_nk=True)
        gws.gws_gated_bwd_x(self.dg, self.du, d["gate"].w_hat, d["up"].w_hat, self.dx, w_is_nk=True)
        for name, grad in (("gate", self.dg), ("up", self.du)):
            gws.gws_linear_bwd_w_act8(self.x8, grad, d[name], step, self.workspace, w_is_nk=True)
        return self.dx

    def descend(self, rate):
        for name, w in self.master.items():
            w -= rate * self.desc[name].dw
            self.desc[name].w.copy_(w)

    def token(self, x):
        """Serving: x [1 x width] through the weights as they were last sampled; nothing is kept."""
        h, y = bf16(1, self.F), bf16(1, self.K)
        gws.gws_gated_fwd(x, self.desc["gate"].w_hat, self.desc["up"].w_hat, h, w_is_nk=True)
        gws.gws_gemm_bf16(h, self.desc["down"].w_hat, y, w_is_nk=True)
        return y


def train(tokens, width, block, steps, rate=0.2, say=print):
    """Losses of the steps, and the block."""
    teacher, ffn = GatedFFN(tokens, width, block, seed=1), GatedFFN(tokens, width, block, seed=2)
    for name in ("gate", "up", "down"):                       # the teacher, disturbed
        ffn.master[name] = 0.8 * teacher.master[name] + 0.3 * ffn.master[name]
        ffn.desc[name].w.copy_(ffn.master[name])
    teacher.sample(0)
    gen = torch.Generator(device=DEV).manual_seed(3)
    x = torch.randn(tokens, width, generator=gen, device=DEV).bfloat16()
    goal = teacher.forward(x).float().clone()
    losses = []
    for step in range(1, steps + 1):
        ffn.sample(step)
        error = ffn.forward(x).float() - goal
        losses.append(float((error ** 2).mean() / (goal ** 2).mean()))
        dy = (error * (2.0 / tokens)).bfloat16()              # of the loss summed over columns, averaged over tokens
        ffn.backward(dy, step)
        ffn.descend(rate)
        say(f"step {step}: relative error {losses[-1]:.4f}, mean |dL/db_t| of the gate {ffn.desc['gate'].dbt.abs().mean():.2e}")
    return losses, ffn, x


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=8192)
    ap.add_argument("--width", type=int, default=2048)
    ap.add_argument("--block", type=int, default=5632)
    ap.add_argument("--steps", type=int, default=20)
    a = ap.parse_args()
    losses, ffn, x = train(a.tokens, a.width, a.block, a.steps)
    bits = 8 + 8 / 32
    print(f"kept between the passes: {(a.tokens * (2 * a.block + a.width)) * bits / 8 / 2**20:.0f} MiB, as BF16 {(a.tokens * (2 * a.block + a.width)) * 2 / 2**20:.0f}")
    print("one token:", ffn.token(x[:1])[0, :4].tolist())


if __name__ == "__main__":
    main()
