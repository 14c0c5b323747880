"""Learns a gate over tokens: every operator of the token section of the library in one training step.

    python -m paper_2308_10037_b200.examples.token_gate --steps 200

Tokens are looked up in a learned table (``lr_embed``), a gate sends every token to k of E experts (``lr_route``), and each
expert answers with one learned logit; a token's answer is the weighted sum of its experts' logits, held against a 0/1 target
with the log-loss of the binary model.  Backward, the routing weights' gradient goes to the gate's logits (``lr_route_grad``), the
gate's own gradient comes from the rows kept in 8 bits (``lr_ckpt8_save``, ``lr_ckpt8_grad``), and the table's from the rows'
gradient summed over the places of each token (``lr_embed_grad``).  The targets are planted: half of the tokens are positive,
with a tenth of the targets flipped, so the loss can fall to about 0.33 and no further.  A bias per expert, moved a little
against the load after every step, spreads the tokens over the experts.  At the end a logistic model is fitted on the learned rows
with ``lr_fit`` and scored with ``lr_predict``, as on any other matrix of rows.
"""
from __future__ import annotations

import argparse

import torch

from paper_2308_10037_b200 import api, build


class TokenGate:
    """Table [V, n], gate W [E, n] and b [E], one logit a [E] per expert; all float32."""

    def __init__(self, vocab, n, experts, k, ctx, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.ctx, self.k, self.vocab, self.scale = ctx, k, vocab, n ** 0.5
        self.table = torch.randn(vocab, n, generator=g, device="cuda") / self.scale
        self.W = torch.randn(experts, n, generator=g, device="cuda") / n ** 0.5
        self.b = torch.zeros(experts, device="cuda")
        self.a = 0.1 * torch.randn(experts, generator=g, device="cuda")
        self.balance = torch.zeros(experts, device="cuda")

    def forward(self, tokens):
        X = self.ctx.embed(self.table, tokens, self.scale)
        logits = torch.addmm(self.b, X, self.W.t())
        ids, w, counts = self.ctx.route(logits, self.k, bias=self.balance, score="sigmoid")
        z = (w * self.a[ids.long()]).sum(1)
        return X, logits, ids, w, counts, z

    def step(self, tokens, y):
        """Loss, expert counts and the gradients of (table, W, b, a) at the current parameters."""
        X, logits, ids, w, counts, z = self.forward(tokens)
        q, s = self.ctx.ckpt8_save(X)               # from here on the rows are kept in a quarter of their bytes
        del X
        loss = torch.nn.functional.binary_cross_entropy_with_logits(z, y)
        dz = (torch.sigmoid(z) - y) / len(y)
        chosen = ids.long()
        da = torch.zeros_like(self.a).index_add_(0, chosen.flatten(), (dz[:, None] * w).flatten())
        dlogits = self.ctx.route_grad(logits, ids, (dz[:, None] * self.a[chosen]).contiguous(), score="sigmoid")
        dW, db = self.ctx.ckpt8_grad(q, s, dlogits)
        dtable = self.ctx.embed_grad(tokens, dlogits @ self.W, self.vocab, self.scale)
        return loss, counts, (dtable, dW, db, da)


def train(steps, batch=4096, vocab=2000, n=64, experts=16, k=2, lr=2.0, seed=0, ctx=None, say=None):
    """Trains for ``steps`` steps; returns (model, losses, counts of the last step, tokens' planted labels)."""
    ctx = ctx or api.Context()
    model = TokenGate(vocab, n, experts, k, ctx, seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    positive = (torch.rand(vocab, generator=g, device="cuda") < 0.5).float()
    losses, counts = [], None
    for i in range(steps):
        tokens = torch.randint(0, vocab, (batch,), generator=g, device="cuda")
        flipped = (torch.rand(batch, generator=g, device="cuda") < 0.1).float()
        y = (positive[tokens] - flipped).abs()
        loss, counts, grads = model.step(tokens, y)
        for p, d, rate in zip((model.table, model.W, model.b, model.a), grads, (20 * lr, lr, lr, 5 * lr)):
            p.sub_(d, alpha=rate)
        model.balance.add_(torch.sign(counts.float().mean() - counts.float()), alpha=0.002)
        losses.append(loss)
        if say and (i % max(1, steps // 10) == 0 or i == steps - 1):
            say(f"step {i:4d}  loss {loss.item():.4f}  busiest expert {counts.max().item() / counts.float().mean().item():.2f} x the mean")
    return model, torch.stack(losses), counts, positive


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--batch", type=int, default=4096, help="tokens per step")
    ap.add_argument("--vocab", type=int, default=2000)
    ap.add_argument("--width", type=int, default=64, help="columns of a row")
    ap.add_argument("--experts", type=int, default=16)
    ap.add_argument("--k", type=int, default=2)
    args = ap.parse_args()
    if not torch.cuda.is_available():
        raise SystemExit("needs a CUDA device: the library has no CPU path")
    build.build()
    ctx = api.Context()
    model, losses, counts, positive = train(args.steps, args.batch, args.vocab, args.width, args.experts, args.k, ctx=ctx, say=print)
    rows = ctx.embed(model.table, torch.arange(args.vocab, device="cuda"), model.scale)
    w, b = api.lr_fit(rows, positive, lr=0.5, iters=200, ctx=ctx)
    f1 = ctx.f1_counts(api.lr_predict(rows, w, b, 0.5, ctx=ctx), positive)[0]
    print(f"loss {losses[0].item():.4f} -> {losses[-1].item():.4f}; a logistic model on the learned rows: f1 {f1:.4f}")
    assert ctx.device_status() == 0
    ctx.close()


if __name__ == "__main__":
    main()
