"""A compressed model distilled from the model it was made from, which then verifies
what it drafts.

The teacher maps a token's embedding through a dense projection W and a vocabulary head.
The student has W as BSQ codes, and a low-rank adapter that trains (Section III-F):

  ids, top, norm     bsq_top_logits, of the teacher's logits
  y0 = X W_hat^T     bsq_gemm, on the codes;  y = y0 + s B (A x)  bsq_adapters_apply
  loss, lse, kept    bsq_distill_loss, through the frozen head
  dy                 bsq_distill_grad
  dA, dB             bsq_adapters_grad;  clip, then SGD  bsq_grad_clip

Afterwards the student drafts a few tokens of every sequence, one after another, the
teacher scores them in one pass, and bsq_draft_verify says which stand and what follows.

  python examples/distill_draft.py [--steps 30]
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


class Pair:
    """A teacher and the student made from it."""

    def __init__(self, d=512, vocab=3000, rank=16, K=32, tau=2.0, seed=1, device="cuda"):
        self.dev, self.K, self.scale, self.vocab = torch.device(device), K, 1.0 / tau, vocab
        self.cfg = bsq.Config(stages=1)
        decs = synth.decoder_params(self.cfg.kind, self.cfg.d, self.cfg.b, self.cfg.hidden, self.cfg.stages, seed=seed)
        self.codec = bsq.bsq_codec_prepare(self.cfg, decs, device=self.dev)
        self.W, _ = synth.weight(d, d, seed=seed, k_outliers=self.cfg.k(d), dtype=torch.bfloat16, device=self.dev)
        self.layer = bsq.bsq_encode(self.cfg, self.codec, self.W)
        g = torch.Generator().manual_seed(seed)
        rn = lambda *s: torch.randn(s, generator=g).to(self.dev)  # noqa: E731
        # embeddings of a size that makes the teacher's logits some units wide
        size = float(self.W.float().square().sum(1).mean().sqrt())
        self.embed = (rn(vocab, d) / size).bfloat16()
        self.head = (rn(vocab, d) * (3.0 / d ** 0.5)).bfloat16()
        self.A, self.B = rn(1, rank, d) / d ** 0.5, torch.zeros((1, d, rank), device=self.dev)
        self.dA, self.dB = torch.zeros_like(self.A), torch.zeros_like(self.B)
        self.clip = bsq.GradPlan([self.dA, self.dB])
        self.refresh()

    def refresh(self):
        self.pool = bsq.AdapterPool(self.A.bfloat16(), self.B.bfloat16())

    def plan(self, M):
        return bsq.bsq_adapters_plan(torch.zeros(M, dtype=torch.int32, device=self.dev), 1)

    def teacher(self, X):
        """Logits in bf16."""
        return (X @ self.W.T) @ self.head.T

    def student(self, X, plan, keep=False):
        """Hidden states; with keep also the adapter's activations."""
        y0 = bsq.bsq_gemm(self.cfg, self.codec, self.layer, X)
        y, t = bsq.bsq_adapters_apply(plan, self.pool, X, y0, out=y0, keep=keep)
        return (y, t) if keep else y

    def step(self, tokens, ignore, lr=20.0, max_norm=1.0):
        """One SGD step on the tokens that are not ignored; their mean divergence and the gradient norm (on the GPU)."""
        X = self.embed[tokens]
        ids, top, norm = bsq.bsq_top_logits(self.teacher(X), self.K, scale=self.scale)
        ids = torch.where(ignore[:, None], -1, ids)
        plan = self.plan(len(tokens))
        y, t = self.student(X, plan, keep=True)
        loss, lse, kept = bsq.bsq_distill_loss(y, self.head, ids, top, norm=norm, scale=self.scale, keep=True)
        live = (~ignore).float()
        g = live / live.sum()
        dy, _ = bsq.bsq_distill_grad(y, self.head, ids, top, lse, g, norm=norm, scale=self.scale, kept=kept, head=False)
        bsq.bsq_adapters_grad(plan, self.pool, X, t, dy, want_dx=False, grads=(self.dA, self.dB))
        stats = bsq.bsq_grad_clip(self.clip, max_norm)
        self.A.add_(self.dA, alpha=-lr)
        self.B.add_(self.dB, alpha=-lr)
        self.refresh()
        return (loss * g).sum(), stats[0]

    def draft(self, last, L, gen):
        """L tokens that the student says after `last` [B]: (tokens [B, L], their logits [B, L, vocab])."""
        plan, tokens, logits = self.plan(len(last)), [], []
        for _ in range(L):
            z = self.student(self.embed[last], plan) @ self.head.T
            r = torch.rand(len(last), generator=gen).to(self.dev)
            none = torch.empty((len(last), 0), device=self.dev)
            _, out = bsq.bsq_draft_verify(z[:, None], none.int(), none, r)  # (nothing drafted: one draw each)
            last = out[:, 0].long()
            tokens.append(out[:, 0])
            logits.append(z)
        return torch.stack(tokens, 1), torch.stack(logits, 1)

    def decode(self, last, L, gen):
        """Draft and verify once: what bsq_draft_verify took and gave."""
        tokens, draft = self.draft(last, L, gen)
        seen = torch.cat([last[:, None], tokens.long()], 1)
        target = self.teacher(self.embed[seen].flatten(0, 1)).view(len(last), L + 1, self.vocab)
        u, r = torch.rand((len(last), L), generator=gen).to(self.dev), torch.rand(len(last), generator=gen).to(self.dev)
        count, out = bsq.bsq_draft_verify(target, tokens, u, r, draft=draft)
        return (target, tokens, u, r, draft), (count, out)


def batch(pair, M=600, seed=2):
    """Tokens, every fifth ignored."""
    g = torch.Generator().manual_seed(seed)
    tokens = torch.randint(0, pair.vocab, (M,), generator=g).to(pair.dev)
    return tokens, (torch.arange(M, device=pair.dev) % 5 == 0)


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=30)
    args = ap.parse_args()
    pair = Pair()
    tokens, ignore = batch(pair)
    gen = torch.Generator().manual_seed(3)
    last = torch.arange(16, device=pair.dev)
    for when in ("before", "after"):
        taken = sum(int(pair.decode(last + 16 * i, 4, gen)[1][0].sum()) for i in range(8))
        print(f"{when} distillation: {taken} of {8 * 16 * 4} drafted tokens stand", flush=True)
        for i in range(args.steps if when == "before" else 0):
            loss, norm = pair.step(tokens, ignore)
            if i % 5 == 0 or i == args.steps - 1:
                print(f"step {i}: divergence {float(loss):.4f}, gradient norm {float(norm):.4f}", flush=True)


if __name__ == "__main__":
    main()
