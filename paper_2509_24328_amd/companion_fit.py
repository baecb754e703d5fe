"""Fits a small companion to a target's answers while the target serves: speculative-sampling
verification emits tokens, their log-probabilities (with alternatives) are what a client gets, and the
same tokens are the companion's training data.

S and A tell how likely the target accepts a drafted token as far as the companion is like the target
(arxiv 2509.24328, Sec. 4.2), and one way to get such a companion is to fit it.  Per step:

  * serve:   the draft proposes k tokens per sequence, sv_verify_sample emits the accepted ones and one
             more, sv_token_logprobs scores what was emitted under the target;
  * fit:     sv_embedding of the emitted tokens' contexts, the companion's body, logits,
             sv_token_logprobs_grad (negative log-likelihood, optionally with an entropy term) in
             place of the logits, the products' gradients, sv_embedding_grad on top of the output
             projection's gradient (tied weights), sv_clip_grad_norm, a step of plain gradient
             descent with momentum.

All three models are first-order here: embedding row of the last token (scaled by sqrt(D)), one tanh
layer, output projection tied to the embedding.  The target and the draft are frozen and random, the
draft a noisy copy of the target.  Only the body's products are torch's; they stand in for a model.

Run:  python -m paper_2509_24328_amd.companion_fit [--steps 200] [--vocab 512]
"""
from __future__ import annotations

import argparse
import json
import math

import torch

from .binding import (SV_F32, alloc_workspace, sv_clip_grad_norm, sv_embedding, sv_embedding_grad,
                      sv_embedding_grad_workspace_bytes, sv_grad_norm_workspace_bytes, sv_row_stats, sv_token_logprobs,
                      sv_token_logprobs_grad, sv_verify_sample)


class Model:
    """Embedding [V, D], one layer [D, D], tied output projection; float32."""

    def __init__(self, V, D, gen, scale=0.5):
        dev = "cuda"
        self.V, self.D, self.scale = V, D, math.sqrt(D)
        self.table = scale / math.sqrt(D) * torch.randn((V, D), generator=gen, device=dev)
        self.layer = torch.randn((D, D), generator=gen, device=dev) / math.sqrt(D)
        self.gain = 6.0

    def noisy(self, amount, gen):
        m = Model.__new__(Model)
        m.__dict__.update(self.__dict__)
        m.table = self.table + amount * self.table.std() * torch.randn(self.table.shape, generator=gen, device="cuda")
        return m

    def body(self, tokens):
        x = torch.empty((tokens.numel(), self.D), device="cuda")
        sv_embedding(self.table, tokens, x, scale=self.scale)
        return x, torch.tanh(x @ self.layer)

    def logits(self, tokens):
        _, h = self.body(tokens)
        return self.gain * (h @ self.table.t())


class Fit:
    """A companion in training: its parameters, gradients, momentum and the scratch of the calls."""

    def __init__(self, model, rows, lr=0.1, momentum=0.9, max_norm=1.0, entropy_weight=0.0):
        self.model, self.lr, self.momentum, self.max_norm = model, lr, momentum, max_norm
        self.params = [model.table, model.layer]
        self.velocity = [torch.zeros_like(p) for p in self.params]
        self.grads = [torch.empty_like(p) for p in self.params]
        f32 = lambda *s: torch.empty(s, device="cuda")
        self.logprob, self.norm, self.g_logprob = f32(rows), f32(1), f32(rows)
        self.g_entropy = None
        self.entropy_weight = entropy_weight
        n = max(sv_embedding_grad_workspace_bytes(rows, model.V, model.D), sv_grad_norm_workspace_bytes(2))
        self.ws = torch.empty(n, dtype=torch.uint8, device="cuda")

    def gradients(self, contexts, tokens):
        """Fills grads with those of the mean negative log-likelihood of tokens (-1: none) after their contexts."""
        m = self.model
        x, h = m.body(contexts)
        z = m.gain * (h @ m.table.t())
        count = (tokens >= 0).sum().clamp(min=1)
        self.g_logprob.copy_((-1.0 / count).expand_as(self.g_logprob))
        if self.entropy_weight:
            self.g_entropy = self.g_logprob * self.entropy_weight
        sv_token_logprobs_grad(z, tokens, self.g_logprob, z, g_entropy=self.g_entropy, logprob=self.logprob)
        dz = z.mul_(m.gain)                                # (in place: z holds the gradient now)
        torch.mm(dz.t(), h, out=self.grads[0])             # output projection ...
        da = (dz @ m.table) * (1 - h * h)
        torch.mm(x.t(), da, out=self.grads[1])
        sv_embedding_grad(da @ m.layer.t(), contexts, self.grads[0], scale=m.scale, accumulate=True, ws=self.ws)   # ... and lookup

    def step(self, contexts, tokens):
        self.gradients(contexts, tokens)
        sv_clip_grad_norm(self.grads, self.max_norm, self.norm, ws=self.ws)
        for p, g, v in zip(self.params, self.grads, self.velocity):
            v.mul_(self.momentum).add_(g)
            p.sub_(v, alpha=self.lr)


def run(V=512, D=32, B=64, k=4, steps=200, seed=0, n_top=5, lr=0.1, noise=0.5, entropy_weight=0.0):
    """List of per-step dicts: similarity of companion and target (S of sv_row_stats), mean log-probability of the
    emitted tokens under the target and under the companion, accepted drafts per sequence, gradient norm."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    target = Model(V, D, gen, scale=1.0)
    draft = target.noisy(noise, gen)
    fit = Fit(Model(V, D, gen), B * (k + 1), lr=lr, entropy_weight=entropy_weight)
    ws = alloc_workspace(B, k, V, SV_F32)
    f32 = lambda *s: torch.empty(s, dtype=torch.float32, device="cuda")
    i32 = lambda *s: torch.empty(s, dtype=torch.int32, device="cuda")
    tokens, n_acc, flags, rank = i32(B, k + 1), i32(B), i32(B), i32(B, k + 1)
    lse_t, lse_c, S, A = (f32(B, k) for _ in range(4))
    logprob, entropy, top_token, top_logprob = f32(B, k + 1), f32(B, k + 1), i32(B, k + 1, n_top), f32(B, k + 1, n_top)
    last = torch.randint(0, V, (B,), generator=gen, device="cuda", dtype=torch.int32)
    log = []
    for step in range(steps):
        contexts = i32(B, k + 1)
        contexts[:, 0] = last
        z_d = f32(B, k, V)
        for i in range(k):                                 # the draft, token by token
            z_d[:, i] = draft.logits(contexts[:, i].contiguous())
            contexts[:, i + 1] = torch.multinomial(torch.softmax(z_d[:, i], -1), 1, generator=gen)[:, 0]
        x = contexts[:, 1:].contiguous()
        z_t = target.logits(contexts.view(-1)).view(B, k + 1, V)
        sv_verify_sample(z_t, None, z_d, x, None, seed, step, tokens, n_acc, flags, None, ws)
        sv_token_logprobs(z_t, tokens, logprob, None, entropy, rank, top_token, top_logprob)

        z_c = fit.model.logits(contexts.view(-1)).view(B, k + 1, V)
        sv_row_stats(z_t[:, :k].contiguous(), z_c[:, :k].contiguous(), x, lse_t, lse_c, S, A, ws=ws)
        fit.step(contexts.view(-1), tokens.view(-1))

        emitted = (n_acc + 1).sum()
        log.append(dict(similarity=float(S.mean()), target=float(logprob.sum() / emitted),
                        companion=float(fit.logprob.sum() / emitted), accepted=float(n_acc.float().mean()),
                        norm=float(fit.norm)))
        last = tokens.gather(1, n_acc.long()[:, None])[:, 0].contiguous()
    return log


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--vocab", type=int, default=512)
    ap.add_argument("--entropy", type=float, default=0.0, help="weight of the entropy term")
    a = ap.parse_args()
    log = run(V=a.vocab, steps=a.steps, entropy_weight=a.entropy)
    for i in sorted({0, len(log) // 4, len(log) // 2, len(log) - 1}):
        print(json.dumps(dict(step=i, **{n: round(v, 4) for n, v in log[i].items()})))


if __name__ == "__main__":
    main()
