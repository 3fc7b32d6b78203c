"""A small language model trained with EfQAT through the library's calls alone.

    python -m paper_2411_11038_b200.lm_step [--steps 30] [--blocks 4] [--no-checkpoint]

Blocks of layer norm -> quantized linear -> GELU -> quantized linear with a residual connection, a final layer norm
and a softmax cross entropy over the vocabulary.  What the backward needs of a block is its two 8-bit activation
checkpoints (the norm's input and the GELU's input) and the norm's statistics: the inputs of the two quantized layers
are formed again from them, so every other activation lives in buffers that all blocks share.  With
checkpoint=False the block keeps the activations themselves.  As everywhere in this package the host code only
orders calls and owns memory; torch adds the residuals and applies the plain SGD of norms and output matrix.
"""
from __future__ import annotations

import argparse

import torch

from . import binding as B


class Block:
    """x + down(gelu(up(norm(x)))), both linears fake-quantized, a fraction of their channels unfrozen."""

    def __init__(self, ctx: B.Context, M: int, D: int, F: int, gen: torch.Generator, checkpoint: bool, first=None,
                 bits: int = 8):
        dev, bf = "cuda", torch.bfloat16
        self.ctx, self.checkpoint, self.D, self.F = ctx, checkpoint, D, F
        normal = lambda n, k, std: (torch.randn((n, k), generator=gen) * std).to(dev)
        self.W = [normal(F, D, D ** -0.5), normal(D, F, 0.5 * F ** -0.5)]
        self.mom = [torch.zeros_like(w) for w in self.W]
        self.bias = [torch.zeros(F, device=dev), torch.zeros(D, device=dev)]
        self.gamma, self.beta = torch.ones(D, device=dev), torch.zeros(D, device=dev)
        self.s_w = [B.init_weight_scales(ctx, w, bits) for w in self.W]
        self.s_x = self.z_x = None                        # MinMax of the first batch
        shared = first if checkpoint else None            # with checkpoints the blocks share their output buffers
        self.norm = B.LayerNormPlan(ctx, M, D, bf, dev, outputs=shared.norm if shared else None)
        self.act = shared.act if shared else B.GeluPlan(ctx, M, F, bf, dev)
        plan = lambda n, k, src: B.LayerPlan(ctx, M, n, k, bf, bits, bits, False, n, dev, outputs=src, ws=src.ws if src else None)
        self.lin = [plan(F, D, shared.lin[0] if shared else None), plan(D, F, shared.lin[1] if shared else None)]
        self.kept = [B.Checkpoint(ctx, M, D, dev), B.Checkpoint(ctx, M, F, dev)] if checkpoint else [None, None]
        self.x = None

    def _quantizers(self, i: int, X: torch.Tensor):
        if self.s_x is None:
            self.s_x, self.z_x = [None, None], [None, None]
        if self.s_x[i] is None:
            self.s_x[i], self.z_x[i] = B.init_act_qparams(self.ctx, X, self.lin[i].spec.x_bits, False)
        return self.s_w[i], self.s_x[i], self.z_x[i]

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        n = self.norm.fwd(x, self.gamma, self.beta, save=self.kept[0])
        h = self.lin[0].fwd(n, self.W[0], *self._quantizers(0, n), self.bias[0])
        a = self.act.fwd(h, save=self.kept[1])
        y = self.lin[1].fwd(a, self.W[1], *self._quantizers(1, a), self.bias[1])
        if not self.checkpoint:
            self.x = x
        return x + y

    def backward(self, dy: torch.Tensor, idx, lr: float) -> torch.Tensor:
        """Gradient of the block's input; idx: the unfrozen channels of the two linears.  The unfrozen rows take
        their SGD step inside the calls."""
        sgd = [B.make_sgd(lr, 0.9, 0.0, w, m) for w, m in zip(self.W, self.mom)]
        kx, kh = self.kept
        a = self.act.recompute(kh) if kh else self.act.y
        self.down = self.lin[1].bwd(dy, a, self.W[1], self.s_w[1], self.s_x[1], self.z_x[1], idx[1], len(idx[1]), sgd=sgd[1])
        dh = self.act.bwd(self.down["dX"], saved=kh) if kh else self.act.bwd(self.down["dX"], x=self.lin[0].Y)
        n = self.norm.recompute(kx, self.gamma, self.beta) if kx else self.norm.y
        self.up = self.lin[0].bwd(dh, n, self.W[0], self.s_w[0], self.s_x[0], self.z_x[0], idx[0], len(idx[0]), sgd=sgd[0])
        self.gn = self.norm.bwd(self.up["dX"], self.gamma, saved=kx) if kx else self.norm.bwd(self.up["dX"], self.gamma, x=self.x)
        dx = dy + self.gn["dx"]
        self.bias[0] -= lr * self.up["db"]
        self.bias[1] -= lr * self.down["db"]
        self.gamma -= lr * self.gn["dgamma"]
        self.beta -= lr * self.gn["dbeta"]
        return dx


class QuantizedLm:
    """Embedding (fixed) -> blocks -> layer norm -> softmax cross entropy; per-layer channel selection every step."""

    def __init__(self, tokens: int, vocab: int, D: int, F: int, blocks: int, unfrozen: float = 0.1,
                 checkpoint: bool = True, seed: int = 0):
        self.ctx = B.Context(0)
        gen = torch.Generator().manual_seed(seed)
        bf = torch.bfloat16
        self.embedding = torch.randn((vocab, D), generator=gen).to(bf).cuda()
        self.head = (torch.randn((vocab, D), generator=gen) * D ** -0.5).cuda()          # fp32 master
        self.head16 = self.head.to(bf)
        self.blocks = []
        for _ in range(blocks):
            self.blocks.append(Block(self.ctx, tokens, D, F, gen, checkpoint, self.blocks[0] if self.blocks else None))
        self.norm = B.LayerNormPlan(self.ctx, tokens, D, bf, "cuda")
        self.gamma, self.beta = torch.ones(D, device="cuda"), torch.zeros(D, device="cuda")
        self.loss = B.LmLossPlan(self.ctx, tokens, vocab, D, "cuda")
        weights = [w for b in self.blocks for w in b.W]
        self.counts = [max(1, B.ratio_to_k(unfrozen, int(w.shape[0]))) for w in weights]
        self.select = B.SelectPlan(self.ctx, B.CWPL, weights, self.counts)

    def kept_bytes(self) -> int:
        """Bytes that the checkpoints of all blocks hold between forward and backward."""
        return sum(k.nbytes for b in self.blocks for k in b.kept if k)

    def step(self, ids: torch.Tensor, labels: torch.Tensor, lr: float) -> torch.Tensor:
        """One training step on tokens `ids` with targets `labels` (int32, negative: none); the mean loss."""
        idx, _, _ = self.select.run()                     # importance + Top-K, per layer
        parts = list(torch.split(idx[:sum(self.counts)], self.counts))
        x = self.embedding[ids]
        for b in self.blocks:
            x = b.forward(x)
        H = self.norm.fwd(x, self.gamma, self.beta)
        per_token = self.loss.fwd(H, self.head16, labels)
        live = labels >= 0
        n = live.sum().clamp(min=1).float()
        mean = per_token.sum() / n
        grads = self.loss.bwd(H, self.head16, labels, live.float() / n)
        out = self.norm.bwd(grads["dH"], self.gamma, x=x)
        dy = out["dx"]
        for i in reversed(range(len(self.blocks))):
            dy = self.blocks[i].backward(dy, parts[2 * i:2 * i + 2], lr)
        self.gamma -= lr * out["dgamma"]
        self.beta -= lr * out["dbeta"]
        self.head -= lr * grads["dW"].float()
        self.head16.copy_(self.head)
        return mean


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--blocks", type=int, default=4)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--vocab", type=int, default=8000)
    ap.add_argument("--dim", type=int, default=512)
    ap.add_argument("--lr", type=float, default=2.0)
    ap.add_argument("--no-checkpoint", action="store_true")
    a = ap.parse_args()
    net = QuantizedLm(a.tokens, a.vocab, a.dim, 4 * a.dim, a.blocks, checkpoint=not a.no_checkpoint)
    gen = torch.Generator().manual_seed(1)
    for k in range(a.steps):
        ids = torch.randint(0, a.vocab, (a.tokens,), generator=gen)
        labels = ((ids * 7 + 3) % a.vocab).to(torch.int32)          # a fixed next token for each token
        loss = net.step(ids.cuda(), labels.cuda(), a.lr)
        if k % 5 == 0 or k + 1 == a.steps:
            print(f"step {k:3d}  loss {float(loss):.4f}", flush=True)
    if net.ctx.device_status():
        raise SystemExit("device status: " + B.status_string(net.ctx.device_status()))
    full = a.tokens * a.dim * 2 * (1 + 1 + 4 + 4) * a.blocks
    print(f"kept between forward and backward: {net.kept_bytes() / 2**20:.1f} MiB in checkpoints"
          f" ({full / 2**20:.1f} MiB as bf16 activations)")


if __name__ == "__main__":
    main()
