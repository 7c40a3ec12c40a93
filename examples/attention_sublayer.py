"""A decoder's self-attention sublayer trained on a packed batch of sentences with 4-bit floating-point weights, then one
more token served against a cache.

    x = scale E[ids] + PE[position],  q | k | v = x Wqkv^T + b,  out = r + D(attention(q, k, v) Wo^T + bo)

Sentences of different lengths lie one after another, without padding: the embedding (mnmt_embed) and the attention
(mnmt_attention_forward) take the rows as they are, the attention with each sentence's start.  The linears are those of
fp4_ffn.py.  Back: dropout, the output projection, the attention's gradients (mnmt_attention_backward) straight into the
gradient of the fused projection, and the table's gradient (mnmt_embed_backward).  Serving appends a key and a value to a
cache and reads it with mnmt_attention_token.

    python examples/attention_sublayer.py [--format mx|nv] [--steps 40]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from fp4_ffn import FORMATS, Linear  # noqa: E402
from paper_2306_04235_gb300 import mnmt  # noqa: E402


def positions(n, d):
    """The sinusoidal table."""
    at = torch.arange(n, dtype=torch.float64)[:, None] / 10000 ** (torch.arange(0, d, 2, dtype=torch.float64) / d)
    return torch.stack([at.sin(), at.cos()], 2).view(n, d).float().cuda()


class Sublayer:
    def __init__(self, d, heads, kv_heads, vocab, lens, fmt="mx", p=0.1, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.d, self.hq, self.hkv, self.dh, self.V, self.p, self.seed, self.step = d, heads, kv_heads, d // heads, vocab, p, seed, 0
        self.starts = [sum(lens[:i]) for i in range(len(lens) + 1)]
        self.T = T = self.starts[-1]
        n = (heads + 2 * kv_heads) * self.dh
        self.table = torch.randn((vocab, d), generator=gen, device="cuda") * d ** -0.5
        self.scale, self.pe = d ** 0.5, positions(max(lens), d)
        self.pos = torch.cat([torch.arange(m, dtype=torch.int32) for m in lens]).cuda()
        self.qkv, self.wo = Linear(n, d, T, FORMATS[fmt], gen), Linear(d, d, T, FORMATS[fmt], gen)
        bf = dict(dtype=torch.bfloat16, device="cuda")
        self.x, self.o, self.gv, self.gqkv = torch.empty((T, d), **bf), torch.empty((T, heads, self.dh), **bf), torch.empty((T, d), **bf), torch.empty((T, n), **bf)
        self.lse = torch.empty((heads, T), device="cuda")
        self.out, self.gr, self.gtable = torch.empty((T, d), device="cuda"), torch.empty((T, d), device="cuda"), torch.empty_like(self.table)
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        start = torch.tensor(self.starts, dtype=torch.int32, device="cuda")
        self.attn = mnmt.AttentionShape(len(lens), T, T, heads, kv_heads, self.dh, mnmt.BF16, True, self.dh ** -0.5, start, start)
        size = max(mnmt.mnmt_attention_forward_workspace(self.attn), mnmt.mnmt_attention_backward_workspace(self.attn),
                   mnmt.mnmt_embed_backward_workspace(T, vocab, d))
        self.ws = torch.empty(size, dtype=torch.uint8, device="cuda")
        # heads of queries, keys and values beside each other, in the projection's output and in its gradient
        split = lambda y: y.view(T, -1, self.dh).split([heads, kv_heads, kv_heads], 1)  # noqa: E731
        (self.q, self.k, self.v), (self.dq, self.dk, self.dv) = split(self.qkv.y), split(self.gqkv)

    def forward(self, ids):
        """Token ids [T] -> the fp32 residual stream [T][d]."""
        self.ids = ids
        self.qkv.pack(), self.wo.pack()
        mnmt.mnmt_embed(ids, self.T, self.table, mnmt.F32, self.d, self.V, self.d, self.scale, self.x, mnmt.BF16, self.d, self.pos, self.pe, self.d,
                        self.pe.shape[0], self.status)
        self.qkv.forward(self.x)
        H = mnmt.heads
        mnmt.mnmt_attention_forward(self.attn, H(self.q), H(self.k), H(self.v), H(self.o), self.lse, self.ws, self.status)
        y = self.wo.forward(self.o.view(self.T, self.d))
        self.r = self.x.float()
        mnmt.mnmt_dropout(y, mnmt.BF16, self.d, self.r, self.d, 1.0, self.p, self.seed, self.step, False, self.T, self.d, self.out, mnmt.F32, self.d)
        return self.out

    def backward(self, g):
        """g: gradient of the output, fp32; those of the weights stay in the layers, the table's in gtable (without the
        residual's own way to it)."""
        mnmt.mnmt_dropout_backward(g, mnmt.F32, self.d, None, mnmt.BF16, self.d, None, 0, 1.0, self.p, self.seed, self.step, False, self.T, self.d, self.gv,
                                   self.d, self.gr, self.d)
        go, H = self.wo.backward(self.gv).view_as(self.o), mnmt.heads
        mnmt.mnmt_attention_backward(self.attn, H(self.q), H(self.k), H(self.v), H(self.o), self.lse, H(go), H(self.dq), H(self.dk), H(self.dv), self.ws,
                                     self.status)
        gx = self.qkv.backward(self.gqkv)
        mnmt.mnmt_embed_backward(self.ids, self.T, gx, mnmt.BF16, self.d, self.scale, -1, self.V, self.d, self.gtable, mnmt.F32, self.d, False, self.ws,
                                 self.status)

    def update(self, lr):
        for lin in (self.qkv, self.wo):
            lin.w.add_(lin.gw, alpha=-lr)
            lin.b.add_(lin.gb, alpha=-lr)
        self.table.add_(self.gtable, alpha=-lr / self.scale)
        self.step += 1


class Cache:
    """Keys and values of one sentence, up to `room` of them, and the attention of the next token."""

    def __init__(self, s, room):
        bf = dict(dtype=torch.bfloat16, device="cuda")
        self.k, self.v = torch.zeros((room, s.hkv, s.dh), **bf), torch.zeros((room, s.hkv, s.dh), **bf)
        self.o, self.n = torch.empty((1, s.hq, s.dh), **bf), torch.zeros(1, dtype=torch.int32, device="cuda")
        start = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.shape = mnmt.AttentionShape(1, 1, room, s.hq, s.hkv, s.dh, mnmt.BF16, False, s.attn.scale, None, start, k_len=self.n)
        self.ws = torch.empty(mnmt.mnmt_attention_token_workspace(self.shape), dtype=torch.uint8, device="cuda")
        self.filled = 0

    def fill(self, k, v):
        n = k.shape[0]
        self.k[self.filled:self.filled + n], self.v[self.filled:self.filled + n] = k, v
        self.filled += n
        self.n.fill_(self.filled)

    def step(self, q, k, v):
        """The context [1][heads][dh] of the next token, whose key and value join the cache."""
        self.fill(k, v)
        H = mnmt.heads
        mnmt.mnmt_attention_token(self.shape, H(q), H(self.k), H(self.v), H(self.o), None, self.ws)
        return self.o


def train(fmt="mx", steps=40, d=256, heads=4, kv_heads=2, vocab=400, lens=(46, 20, 77, 128, 33), lr=2e-4, seed=1):
    """Fits fixed random targets; returns the losses and the trained sublayer."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = Sublayer(d, heads, kv_heads, vocab, list(lens), fmt, 0.1, seed)
    ids = torch.randint(0, vocab, (s.T,), generator=gen, device="cuda", dtype=torch.int32)
    target = torch.randn((s.T, d), generator=gen, device="cuda")
    losses = []
    for _ in range(steps):
        diff = s.forward(ids) - target
        losses.append(float((diff * diff).sum(1).mean()))
        s.backward((2 / s.T) * diff)
        s.update(lr)
    assert int(s.status) == 0 and int(s.qkv.status) == 0 and int(s.wo.status) == 0
    return losses, s


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--format", choices=list(FORMATS), default="mx")
    ap.add_argument("--steps", type=int, default=40)
    args = ap.parse_args()
    losses, s = train(args.format, args.steps)
    cache = Cache(s, 64)
    cache.fill(s.k[:45], s.v[:45])
    o = cache.step(s.q[45:46], s.k[45:46], s.v[45:46])
    print(f"loss {losses[0]:.3f} -> {losses[-1]:.3f} in {len(losses)} steps")
    print(f"served token: largest difference to the prompt's own last row {float((o - s.o[45:46]).abs().max()):.4f}")


if __name__ == "__main__":
    main()
