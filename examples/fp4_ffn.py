"""An FFN sublayer trained with 4-bit floating-point weights and activations, then
served with the same packed weights.

    out = gamma r + D(relu-dropout hidden W2^T + b2),  hidden = D(relu(x W1^T + b1))

Training keeps fp32 master weights and packs them before every step
(mnmt_fp4_quantize); both linears quantise their input in the call
(mnmt_fp4_linear); dropout draws its masks again in the backward pass
(mnmt_dropout, mnmt_dropout_backward); the linears' gradients are straight-through
(mnmt_fp4_linear_backward).  Serving is one token through the packed weights with
ReLU in the epilogue.

    python examples/fp4_ffn.py [--format mx|nv] [--steps 60]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2306_04235_gb300 import mnmt  # noqa: E402

FORMATS = {"mx": mnmt.FP4_MX, "nv": mnmt.FP4_NV}
G_X, G_W = 16 / 2688, 0.5 / 2688  # tensor scales (NV): the largest magnitudes expected, over 6 x 448


def packed(rows, cols, fmt, g):
    """An empty packed matrix."""
    return mnmt.Fp4(rows, cols, fmt, g, torch.empty((rows, mnmt.mnmt_fp4_pitch(cols)), dtype=torch.uint8, device="cuda"),
                    torch.empty(mnmt.mnmt_fp4_scale_bytes(rows, cols, fmt), dtype=torch.uint8, device="cuda"))


class Linear:
    """fp32 master weights, their packed form, and the buffers of a training step of M rows."""

    def __init__(self, n, k, M, fmt, gen):
        self.N, self.K, self.M = n, k, M
        self.w = torch.randn((n, k), generator=gen, device="cuda") * k ** -0.5
        self.b = torch.zeros(n, device="cuda")
        self.wq, self.xq = packed(n, k, fmt, G_W), packed(M, k, fmt, G_X)
        self.y = torch.empty((M, n), dtype=torch.bfloat16, device="cuda")
        self.gx = torch.empty((M, k), dtype=torch.bfloat16, device="cuda")
        self.gw, self.gb = torch.empty_like(self.w), torch.empty_like(self.b)
        self.ws = torch.empty(mnmt.mnmt_fp4_linear_backward_workspace(M, n, k), dtype=torch.uint8, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def pack(self):
        mnmt.mnmt_fp4_quantize(self.wq, self.w, mnmt.F32, self.K)

    def forward(self, x):
        self.x = x
        mnmt.mnmt_fp4_linear(self.xq, self.wq, x, mnmt.BF16, self.K, self.b, False, self.y, mnmt.BF16, self.N, self.status)
        return self.y

    def backward(self, g):
        mnmt.mnmt_fp4_linear_backward(self.xq, self.wq, g, self.N, self.x, mnmt.BF16, self.K, self.w, mnmt.F32, self.K, self.ws,
                                      self.gx, self.K, self.gw, self.K, self.gb, self.status)
        return self.gx


class FfnSublayer:
    def __init__(self, d, F, M, fmt="mx", p=0.1, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.d, self.F, self.M, self.p, self.seed, self.step = d, F, M, p, seed, 0
        self.w1, self.w2 = Linear(F, d, M, FORMATS[fmt], gen), Linear(d, F, M, FORMATS[fmt], gen)
        self.gamma = 1.0
        bf = dict(dtype=torch.bfloat16, device="cuda")
        self.h, self.gu, self.gv = torch.empty((M, F), **bf), torch.empty((M, F), **bf), torch.empty((M, d), **bf)
        self.out, self.gr = torch.empty((M, d), device="cuda"), torch.empty((M, d), device="cuda")
        self.ggamma = torch.empty(1, device="cuda")
        self.ws = torch.empty(mnmt.DROPOUT_WORKSPACE, dtype=torch.uint8, device="cuda")

    def forward(self, x, r):
        """x [M][d] bf16, the residual stream r [M][d] fp32 -> fp32 [M][d]."""
        self.r = r
        self.w1.pack()
        self.w2.pack()
        u = self.w1.forward(x)
        # two dropouts a step, each with an offset of its own
        mnmt.mnmt_dropout(u, mnmt.BF16, self.F, None, 0, 1.0, self.p, self.seed, 2 * self.step, True, self.M, self.F, self.h, mnmt.BF16, self.F)
        v = self.w2.forward(self.h)
        mnmt.mnmt_dropout(v, mnmt.BF16, self.d, r, self.d, self.gamma, self.p, self.seed, 2 * self.step + 1, False, self.M, self.d, self.out,
                          mnmt.F32, self.d)
        return self.out

    def backward(self, g):
        """g: gradient of the output, fp32 -> gradients of x (bf16) and r (fp32); those of the weights stay in the layers."""
        mnmt.mnmt_dropout_backward(g, mnmt.F32, self.d, None, mnmt.BF16, self.d, self.r, self.d, self.gamma, self.p, self.seed,
                                   2 * self.step + 1, False, self.M, self.d, self.gv, self.d, self.gr, self.d, self.ggamma, self.ws)
        gh = self.w2.backward(self.gv)
        mnmt.mnmt_dropout_backward(gh, mnmt.BF16, self.F, self.w1.y, mnmt.BF16, self.F, None, 0, 1.0, self.p, self.seed, 2 * self.step, True,
                                   self.M, self.F, self.gu, self.F)
        return self.w1.backward(self.gu), self.gr

    def update(self, lr):
        for lin in (self.w1, self.w2):
            lin.w.add_(lin.gw, alpha=-lr)
            lin.b.add_(lin.gb, alpha=-lr)
        self.gamma -= lr * float(self.ggamma)
        self.step += 1

    def serve(self, x, r):
        """A few tokens (x [m][d] bf16, r [m][d] fp32) through the packed weights: no dropout, one launch per linear."""
        m, f = x.shape[0], self.w1.wq.format
        h = torch.empty((m, self.F), dtype=torch.bfloat16, device="cuda")
        v = torch.empty((m, self.d), dtype=torch.float32, device="cuda")
        mnmt.mnmt_fp4_linear(packed(m, self.d, f, G_X), self.w1.wq, x, mnmt.BF16, self.d, self.w1.b, True, h, mnmt.BF16, self.F)
        mnmt.mnmt_fp4_linear(packed(m, self.F, f, G_X), self.w2.wq, h, mnmt.BF16, self.F, self.w2.b, False, v, mnmt.F32, self.d)
        return r * self.gamma + v


def train(fmt="mx", steps=60, d=256, F=1024, M=512, p=0.1, lr=0.01, seed=1):
    """Fits a fixed random FFN; returns the losses and the trained sublayer with one batch."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((M, d), generator=gen, device="cuda").to(torch.bfloat16)
    r = torch.randn((M, d), generator=gen, device="cuda") * 0.1
    a, b = torch.randn((F, d), generator=gen, device="cuda") * d ** -0.5, torch.randn((d, F), generator=gen, device="cuda") * F ** -0.5
    target = r * 0.7 + torch.relu(x.float() @ a.t()) @ b.t()
    layer = FfnSublayer(d, F, M, fmt, p, seed)
    losses = []
    for _ in range(steps):
        diff = layer.forward(x, r) - target
        losses.append(float((diff * diff).sum(1).mean()))
        layer.backward((2 / M) * diff)
        layer.update(lr)
    assert int(layer.w1.status) == 0 and int(layer.w2.status) == 0
    return losses, layer, x, r, target


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--format", choices=list(FORMATS), default="mx")
    ap.add_argument("--steps", type=int, default=60)
    args = ap.parse_args()
    losses, layer, x, r, target = train(args.format, args.steps)
    layer.w1.pack(), layer.w2.pack()
    one = layer.serve(x[:1], r[:1])
    print(f"loss {losses[0]:.3f} -> {losses[-1]:.3f} in {len(losses)} steps, gamma {layer.gamma:.3f}")
    print(f"served token: squared error {float(((one - target[:1]) ** 2).sum()):.3f}")


if __name__ == "__main__":
    main()
