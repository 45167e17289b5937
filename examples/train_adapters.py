"""Adapters of several tenants trained beside one compressed projection, then
served together.

A projection's weights are BSQ-encoded once and stay as they are. Each tenant has
its own low-rank adapter. A training step over a batch of all tenants' tokens:

  y0 = X W_hat^T            bsq_gemm, on the codes
  y  = y0 + s B (A x)       bsq_adapters_apply, each token its tenant's
  loss, lse                 bsq_xent_loss, against a frozen vocabulary head
  dy                        bsq_xent_grad
  dA, dB                    bsq_adapters_grad
  clip, then SGD            bsq_grad_clip

and afterwards a decode step of one token per tenant through the same calls.

  python examples/train_adapters.py [--steps 30]
"""
import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2607_08643_amd as bsq  # noqa: E402
import synth  # noqa: E402


class Tenants:
    """One compressed projection, a frozen head, and an adapter per tenant."""

    def __init__(self, d_in=512, d_out=384, vocab=2000, tenants=5, rank=16, seed=1, device="cuda"):
        self.dev, self.rank, self.tenants = torch.device(device), rank, tenants
        self.cfg = bsq.Config()
        decs = synth.decoder_params(self.cfg.kind, self.cfg.d, self.cfg.b, self.cfg.hidden, self.cfg.stages, seed=seed)
        self.codec = bsq.bsq_codec_prepare(self.cfg, decs, device=self.dev)
        W, _ = synth.weight(d_out, d_in, seed=seed, k_outliers=self.cfg.k(d_in), device=self.dev)
        self.layer = bsq.bsq_encode(self.cfg, self.codec, W)
        g = torch.Generator().manual_seed(seed)
        rn = lambda *s: torch.randn(s, generator=g).to(self.dev)  # noqa: E731
        self.head = (rn(vocab, d_out) * 0.05).bfloat16()
        # fp32 masters; the operators read bf16 copies
        self.A = rn(tenants, rank, d_in) / d_in ** 0.5
        self.B = torch.zeros((tenants, d_out, rank), device=self.dev)
        self.scale = torch.full((tenants,), 2.0, device=self.dev)
        self.dA, self.dB = torch.zeros_like(self.A), torch.zeros_like(self.B)
        self.clip = bsq.GradPlan([self.dA, self.dB])
        self.refresh()

    def refresh(self):
        self.pool = bsq.AdapterPool(self.A.bfloat16(), self.B.bfloat16(), self.scale)

    def forward(self, X, plan, keep):
        y0 = bsq.bsq_gemm(self.cfg, self.codec, self.layer, X)
        return bsq.bsq_adapters_apply(plan, self.pool, X, y0, out=y0, keep=keep)

    def step(self, X, ids, target, lr=2.0, max_norm=1.0):
        """One SGD step; the mean loss and the gradient norm (on the GPU)."""
        plan = bsq.bsq_adapters_plan(ids, self.tenants)
        y, t = self.forward(X, plan, keep=True)
        loss, lse = bsq.bsq_xent_loss(y, self.head, target)
        live = (target >= 0).float()
        g = live / live.sum()
        dy, _ = bsq.bsq_xent_grad(y, self.head, target, lse, g, head=False)
        bsq.bsq_adapters_grad(plan, self.pool, X, t, dy, want_dx=False, grads=(self.dA, self.dB))
        stats = bsq.bsq_grad_clip(self.clip, max_norm)
        self.A.add_(self.dA, alpha=-lr)
        self.B.add_(self.dB, alpha=-lr)
        self.refresh()
        return (loss * g).sum(), stats[0]

    def decode(self, X, ids):
        """The next token of each of a few sequences."""
        y, _ = self.forward(X, bsq.bsq_adapters_plan(ids, self.tenants), keep=False)
        loss, lse = bsq.bsq_xent_loss(y, self.head, torch.zeros(len(ids), dtype=torch.int64, device=self.dev))
        logits = y.float() @ self.head.float().T
        return logits.argmax(1), lse


def batch(model, M=600, seed=2):
    """Tokens of the tenants in runs, some of no tenant; prompts without a loss.
    A tenant's words follow from its inputs by a map of its own."""
    g = torch.Generator().manual_seed(seed)
    d_in, d_out = model.A.shape[2], model.B.shape[1]
    X = torch.randn((M, d_in), generator=g).to(model.dev).bfloat16()
    ids = torch.randint(-1, model.tenants, (M // 20 + 1,), generator=g).repeat_interleave(20)[:M].int().to(model.dev)
    maps = torch.randn((model.tenants + 1, d_in, 3), generator=g).to(model.dev)
    kind = torch.einsum("md,mdk->mk", X.float(), maps[(ids + 1).long()]).argmax(1)
    target = kind + 3 * (ids.long() + 1)
    target[::5] = -100
    return X, ids, target


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=30)
    args = ap.parse_args()
    model = Tenants()
    X, ids, target = batch(model)
    for i in range(args.steps):
        loss, norm = model.step(X, ids, target)
        if i % 5 == 0 or i == args.steps - 1:
            print(f"step {i}: loss {float(loss):.4f}, gradient norm {float(norm):.4f}", flush=True)
    words, _ = model.decode(X[:8].contiguous(), ids[:8].contiguous())
    print("next words of eight sequences:", words.tolist())


if __name__ == "__main__":
    main()
