"""One GraphPO training step of a small policy model, end to end on the GPU.

    python examples/policy_step.py [--steps N] [--teacher WEIGHT]

A batch of sampled rollouts (synthetic) gives per-edge advantages (GraphPO.__call__); the model is
a token embedding, one residual layer and a vocabulary head tied to the embedding.  A step embeds the
tokens, runs the layer, takes the sampled next tokens' log-probabilities and entropies from the
head without ever holding its logits (vocab_logp), the policy loss and its gradient (token_loss),
the entropy bonus, the gradients of hidden states and matrix (vocab_grad), the layer's own, and the
embedding's, added to the tied matrix's (embed_grad).  The first step's old log-probabilities are the
model's own.  With a teacher's weight the policy also learns from another policy's top tokens at the same places
(vocab_distill, whose gradients are added to the others: vocab_distill_grad).
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2606_18954_gb300 as P  # noqa: E402
from paper_2606_18954_gb300 import workloads as W  # noqa: E402


class Policy:
    """Embedding E [V, d] (tied to the head), one residual layer x + tanh(x A)."""

    def __init__(self, vocab, d, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.table = (torch.randn(vocab, d, generator=g, device="cuda") * 0.05).bfloat16()
        self.layer = (torch.randn(d, d, generator=g, device="cuda") / d ** 0.5).bfloat16()
        self.scale = d ** 0.5

    def forward(self, gp, ids):
        x = gp.embed(self.table, ids, scale=self.scale)
        t = torch.tanh(x @ self.layer)
        return x, t, x + t

    def backward(self, gp, ids, x, t, d_hidden, d_table):
        """Gradient of the layer; the embedding's is added to `d_table`, the head's."""
        da = d_hidden * (1 - t * t)
        dx = d_hidden + da @ self.layer.t()
        gp.embed_grad(dx, ids, self.table.shape[0], scale=self.scale, out=d_table, accumulate=True)
        return x.t() @ da


def train(steps=3, vocab=5000, d=256, groups=4, lr=0.5, entropy_weight=1e-3, temperature=1.0, seed=0, teacher_weight=0.0, top=16):
    """Runs `steps` optimiser steps on one batch; returns the losses (token_loss's, without the bonus; with a teacher plus its weight
    times the mean divergence from its `top` tokens)."""
    b = W.make_batch(W.CONFIGS["tiny"].scaled(groups=groups))
    gp = P.GraphPO(kappa=b["kappa"], w=b["w"], lambda_eff=b["lambda_eff"])
    batch = P.Batch.from_arrays(b)
    adv = gp(batch, nodes=True)
    gp.check()
    T = batch.total_tokens
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    ids = torch.randint(0, vocab, (T,), generator=g, device="cuda", dtype=torch.int32)      # inputs: the tokens so far
    target = torch.randint(0, vocab, (T,), generator=g, device="cuda", dtype=torch.int32)   # the sampled next ones
    policy = Policy(vocab, d, seed)
    plan = gp.loss_plan(batch)
    old, losses = None, []
    if teacher_weight > 0.0:  # its log-probabilities of its top tokens, once for all steps
        teacher = Policy(vocab, d, seed + 1)
        taught, ids_top = torch.log_softmax(teacher.forward(gp, ids)[2].float() @ teacher.table.float().t(), 1).topk(top, dim=1)
    for _ in range(steps):
        x, t, hidden = policy.forward(gp, ids)
        head = gp.vocab_logp(hidden, policy.table, target, scale=1.0 / temperature, entropy=True)
        old = head["logp"].clone() if old is None else old
        loss = gp.token_loss(batch, plan, head["logp"], old, edge_adv=adv["edge_adv"])
        bonus = torch.full((T,), -entropy_weight / T, device="cuda")                        # of -weight * mean entropy
        grads = gp.vocab_grad(hidden, policy.table, target, head["lse"], loss["grad_logp"], scale=1.0 / temperature,
                              entropy=head["entropy"], grad_entropy=bonus, logp=head["logp"])
        total = loss["loss"]
        if teacher_weight > 0.0:
            far = gp.vocab_distill(hidden, policy.table, ids_top, taught, scale=1.0 / temperature, tail=True)
            share = torch.full((T,), teacher_weight / T, device="cuda")                     # of weight * mean divergence
            more = gp.vocab_distill_grad(hidden, policy.table, ids_top, far["delta"], far["rest"], far["rest_lse"], share,
                                         scale=1.0 / temperature, accumulate=True,          # (the matrix's are added up there)
                                         out={"d_hidden": torch.empty_like(hidden), "d_weight": grads["d_weight"]})
            grads["d_hidden"] += more["d_hidden"]
            total = total + teacher_weight * far["loss"].mean()
        d_layer = policy.backward(gp, ids, x, t, grads["d_hidden"], grads["d_weight"])
        policy.table -= lr * grads["d_weight"]
        policy.layer -= lr * d_layer
        gp.check()
        losses.append(float(total))
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=5)
    ap.add_argument("--teacher", type=float, default=0.0, metavar="WEIGHT")
    a = ap.parse_args()
    for i, v in enumerate(train(steps=a.steps, teacher_weight=a.teacher)):
        print(f"step {i}: loss {v:+.6f}")
