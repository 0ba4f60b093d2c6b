#!/usr/bin/env python3
"""A policy head trained with the operators around the actor step.

Warm start: the head's logits on demonstrations go through pcm_token_logprobs, the gradient of the mean negative
log-probability (less an entropy bonus) comes from pcm_token_logprobs_backward, and pcm_muon_step updates the weights.
Then GRPO on rollouts: pcm_token_logprobs scores the rollouts' tokens under the policy that made them (logp_old, its
entropy and the alternatives it saw as likeliest), the selection and the masked actor step follow, and pcm_muon_step takes
the place of AdamW.

    python examples/warm_start_and_grpo.py [--warm-steps 40] [--grpo-steps 3]
"""
from __future__ import annotations

import argparse
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import numpy as np
import torch

import paper_2605_16154_amd as pcm
from workloads import CONFIGS, make_hidden_numpy, make_rollouts

NAMES = ("Wg", "Wu", "Wd", "Wo")


def logits_of(x, w):
    """The head: gated projections, down projection, logits."""
    return ((torch.nn.functional.silu(x @ w[0]) * (x @ w[1])) @ w[2]) @ w[3]


class Head:
    """fp32 master weights with their momentum, and the bf16 copies that the products read."""

    def __init__(self, d, ff, V, generator, device):
        shapes = ((d, ff), (d, ff), (ff, d), (d, V))
        self.master = [torch.randn(s, generator=generator, device=device) * s[0] ** -0.5 for s in shapes]
        self.momentum = [torch.zeros_like(w) for w in self.master]
        self.bf16 = [w.to(torch.bfloat16) for w in self.master]

    def update(self, grads, lr):
        pcm.pcm_muon_step(grads, self.master, self.momentum, lr=lr, weights_bf16=self.bf16)


def warm_start(head, steps, rows, lr, generator, device, entropy_coef=1e-3):
    """-> the loss of every step.  The demonstrations are the choices of another head."""
    d, V = head.master[0].shape[0], head.master[3].shape[1]
    teacher = Head(d, head.master[0].shape[1], V, generator, device)
    x = torch.randn((rows, d), generator=generator, device=device).to(torch.bfloat16)
    tokens = logits_of(x, teacher.bf16).argmax(dim=1).to(torch.int32)
    ones = torch.ones(rows, device=device) / rows
    losses = []
    for _ in range(steps):
        w = [b.detach().requires_grad_() for b in head.bf16]
        z = logits_of(x, w)
        got = pcm.pcm_token_logprobs(z.detach(), tokens)
        dz = pcm.pcm_token_logprobs_backward(z.detach(), tokens, got["lse"], -ones, entropy=got["entropy"], dentropy=-entropy_coef * ones)
        z.backward(dz)
        head.update([p.grad.float() for p in w], lr)
        losses.append(-got["logp"].mean() - entropy_coef * got["entropy"].mean())
    return [loss.item() for loss in losses]


def grpo(head, cfg, steps, lr, device):
    """-> a dict per step: loss, mean ratio, entropy, share of the tokens that were among the four likeliest."""
    t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(device)
    state = pcm.pcm_state_init(cfg.K, device)
    report = []
    for step in range(steps):
        ro = make_rollouts(cfg, step)
        hidden, tokens = t(make_hidden_numpy(cfg, step)).to(torch.bfloat16), t(ro["tokens"].reshape(-1))
        scored = pcm.pcm_token_logprobs(logits_of(hidden, head.bf16), tokens, top=4)
        C, valid, adv, active = pcm.pcm_score_phases(t(ro["actions"]), t(ro["phase"]), t(ro["reward"]), t(ro["n_chunks"]),
                                                     cfg.n_groups, cfg.G, cfg.K)
        keep = pcm.pcm_update_keep_probs(state, C, valid)
        kept, _, n_kept = pcm.pcm_sample_chunks(keep, t(ro["phase"]), t(ro["n_chunks"]), active, cfg.B, cfg.seed, step)
        out = pcm.grpo_masked_actor_step(hidden, tokens, scored["logp"], adv, kept, n_kept, cfg.T, cfg.N, cfg.A, *head.bf16,
                                         eps_high=0.4, loss_scale=1.0 / cfg.T, want_dX=False)
        head.update([out["d" + k] for k in NAMES], lr)
        among = (scored["top_ids"] == tokens[:, None].int()).any(dim=1).float().mean()
        report.append(dict(loss=out["loss"].item(), ratio=out["stats"][1].item(), entropy=scored["entropy"].mean().item(),
                           among_four=among.item()))
    return report


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--warm-steps", type=int, default=40)
    ap.add_argument("--grpo-steps", type=int, default=3)
    ap.add_argument("--rows", type=int, default=2000)
    ap.add_argument("--lr", type=float, default=0.02)
    args = ap.parse_args(argv)
    device = torch.device("cuda:0")
    generator = torch.Generator(device=device)
    generator.manual_seed(0)
    cfg = CONFIGS["cfg2"].with_(n_groups=2, G=4, N=16, K=4, B=6, d=256, ff=512)
    head = Head(cfg.d, cfg.ff, cfg.V, generator, device)
    losses = warm_start(head, args.warm_steps, args.rows, args.lr, generator, device)
    print(f"warm start: loss {losses[0]:.3f} -> {losses[-1]:.3f}")
    report = grpo(head, cfg, args.grpo_steps, 0.1 * args.lr, device)
    for step, r in enumerate(report):
        print(f"GRPO step {step}: " + ", ".join(f"{k} {v:.4f}" for k, v in r.items()))
    return losses, report


if __name__ == "__main__":
    main()
