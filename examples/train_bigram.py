"""SparseLoCo training from end to end on one GPU, with everything but the model taken from the library.

The model predicts a token from the one before it: embedding (split table T_S + T_perp, section 2.4), one matrix, softmax.  R
replicas train on their own data for H inner steps,

    sparseloco_embedding_lookup -> torch: logits, loss, their gradients -> sparseloco_embedding_grad -> sparseloco_grad_norm
    -> sparseloco_adamw_step, or sparseloco_adamw_step_8bit,

then one outer step brings them together (sparseloco_outer_step_batch) and sparseloco_reproject_embedding puts T_S back into the
compression subspace.

    python examples/train_bigram.py [--eight] [--rounds N]
"""
from __future__ import annotations

import argparse
import os
import sys
from typing import List

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2601_02360_amd import binding as B  # noqa: E402
from paper_2601_02360_amd import workloads as W  # noqa: E402


class Text:
    """Sequences in which every token is followed by one of four, the first of them mostly."""

    def __init__(self, vocab: int, seed: int):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.vocab = vocab
        self.follows = torch.randint(0, vocab, (vocab, 4), generator=g, device="cuda", dtype=torch.int32)
        self.chance = torch.tensor([0.7, 0.1, 0.1, 0.1], device="cuda")

    def batch(self, n: int, g: torch.Generator):
        x = torch.randint(0, self.vocab, (n,), generator=g, device="cuda", dtype=torch.int32)
        which = torch.multinomial(self.chance, n, replacement=True, generator=g)
        return x, self.follows[x.long(), which]


class Replica:
    """One replica's parameters, gradients, moments and error feedback; T_S is tensor 0 of the plan, the matrix tensor 1."""

    def __init__(self, theta: List[torch.Tensor], plan: B.Plan, eight: bool, tokens: int, d: int, seed: int):
        self.theta = [t.clone() for t in theta]
        self.grads = [torch.zeros_like(t) for t in theta]
        self.ef = [torch.zeros_like(t) for t in theta]
        self.b_theta, self.b_grads = plan.bind(self.theta), plan.bind(self.grads)
        if eight:
            self.moments = plan.adamw_8bit_buffers()
        else:
            self.m, self.v = ([torch.zeros_like(t) for t in theta] for _ in range(2))
            self.moments = plan.bind(self.m), plan.bind(self.v)
        self.step_call = B.sparseloco_adamw_step_8bit if eight else B.sparseloco_adamw_step
        self.x = torch.empty(tokens, d, device="cuda")
        self.norm = torch.empty(2, device="cuda")
        self.data = torch.Generator(device="cuda").manual_seed(seed)
        self.step = 0


def inner_step(r: Replica, plan: B.Plan, text: Text, t_perp: torch.Tensor, grad_ws, norm_ws, lr: float) -> torch.Tensor:
    tokens, d = r.x.shape
    scale = d ** 0.5
    ids, target = text.batch(tokens, r.data)
    B.sparseloco_embedding_lookup(r.theta[0], ids, r.x, t_perp=t_perp, scale=scale)
    logits = r.x @ r.theta[1]
    logp = torch.log_softmax(logits, dim=1)
    loss = -logp[torch.arange(tokens, device="cuda"), target.long()].mean()
    d_logits = logp.exp_()
    d_logits[torch.arange(tokens, device="cuda"), target.long()] -= 1.0
    d_logits /= tokens
    torch.mm(r.x.t(), d_logits, out=r.grads[1])
    B.sparseloco_embedding_grad(d_logits @ r.theta[1].t(), ids, r.grads[0], grad_ws, scale=scale)
    B.sparseloco_grad_norm(plan, r.b_grads, r.norm, norm_ws, max_norm=1.0)
    r.step += 1
    r.step_call(plan, r.b_theta, r.b_grads, *r.moments, lr=lr, step=r.step, weight_decay=0.01, grad_scale=r.norm[1:])
    return loss


def train(rounds: int = 12, inner: int = 25, replicas: int = 2, vocab: int = 300, d: int = 64, k: int = 48, tokens: int = 2048,
          lr: float = 3e-3, eight: bool = False, seed: int = 0):
    """Mean loss of each round, and the parameters that all replicas hold at the end."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    theta = [torch.randn(vocab, d, generator=g, device="cuda") * 0.02, torch.randn(d, vocab, generator=g, device="cuda") * 0.1]
    t_perp, u, coeff = torch.zeros(vocab, d, device="cuda"), W.orthonormal_basis(d, k, seed, "cuda"), torch.empty(vocab * k, device="cuda")
    B.sparseloco_reproject_embedding(theta[0], t_perp, u, coeff)          # T_S + T_perp = the embedding, T_S in Col(U)
    plan = B.Plan([t.shape for t in theta], kappa=1024, quant=False)
    text = Text(vocab, seed + 1)
    group = [Replica(theta, plan, eight, tokens, d, seed + 10 + r) for r in range(replicas)]
    grad_ws, norm_ws = B.embedding_grad_workspace(tokens, vocab, d), B.grad_norm_workspace()
    outer = plan.bind(theta)
    local, ef = plan.bind([r.theta for r in group]), plan.bind([r.ef for r in group])
    messages = plan.bind_messages(*zip(*(plan.message_buffers() for _ in group)))
    losses = []
    for _ in range(rounds):
        losses.append(torch.stack([inner_step(r, plan, text, t_perp, grad_ws, norm_ws, lr) for _ in range(inner) for r in group]).mean())
        B.sparseloco_outer_step_batch(plan, outer, local, ef, messages, 0.95, 1.0)
        B.sparseloco_reproject_embedding(theta[0], t_perp, u, coeff)
        for r in group:
            for mine, shared in zip(r.theta, theta):
                mine.copy_(shared)
    return [x.item() for x in losses], theta, t_perp


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--eight", action="store_true", help="moments in 8 bits")
    ap.add_argument("--rounds", type=int, default=12)
    a = ap.parse_args()
    for i, loss in enumerate(train(rounds=a.rounds, eight=a.eight)[0]):
        print("round %2d  loss %.4f" % (i + 1, loss), flush=True)
