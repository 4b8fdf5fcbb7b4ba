"""Train a small language model on replicas whose embedding, matrices and other tensors each have their own step.

Two replicas of a next-token model on one GPU: an embedding, two hidden matrices, an output matrix.  Rows of the embedding
come from fr_embed_lookup, its gradient from fr_embed_grad; after one clip record over all gradients fr_muon_step updates the
hidden matrices by orthogonalised momentum and fr_adamw_step the embedding and the output matrix.  All of it gives the same
bits on both replicas, so that one can be restored from the other (train_and_recover.py shows that); their fingerprints are
compared after every step.

    python examples/train_language_model.py [--steps 60]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2509_03047_gb300 import flashrec as fr  # noqa: E402

VOCAB, DIM, CONTEXT, HIDDEN = 97, 32, 8, 256
SHAPES = [(VOCAB, DIM), (CONTEXT * DIM, HIDDEN), (HIDDEN, HIDDEN), (HIDDEN, VOCAB)]  # embedding, hidden, hidden, output
MATRICES, OTHERS = (1, 2), (0, 3)
BATCH = 256  # per replica


class Replica:
    def __init__(self, masters):
        self.masters = [x.clone() for x in masters]
        self.weights = [x.bfloat16() for x in masters]
        self.grads = [torch.zeros_like(x) for x in self.weights]
        self.m, self.v = ([torch.zeros_like(x) for x in masters] for _ in range(2))

        def some(which, *lists):
            return [[x[i] for i in which] for x in lists]

        self.all = fr.OptPlan(grads=self.grads)  # for the norm of all gradients
        w, g, p, m, v = some(OTHERS, self.weights, self.grads, self.masters, self.m, self.v)
        self.adamw = fr.OptPlan(w, g, m, v, masters=p)
        w, g, p, m = some(MATRICES, self.weights, self.grads, self.masters, self.m)
        self.muon = fr.MuonPlan(w, g, m, masters=p, update_scale=[0.2 * max(x.shape) ** 0.5 for x in w])
        self.embed = fr.EmbedPlan(VOCAB, DIM, BATCH * CONTEXT)
        self.record = self.all.new_clip()
        self.plan = fr.Plan(self.weights + self.masters + self.m + self.v, 64 << 10)

    def differentiate(self, tokens, target):
        """(loss, gradients) on this replica's part of the batch."""
        w = [t.detach().requires_grad_() for t in self.weights[1:]]
        rows = self.embed.lookup(self.weights[0], tokens).requires_grad_()
        h = torch.relu(rows.flatten(1) @ w[0])
        h = torch.relu(h @ w[1])
        loss = torch.nn.functional.cross_entropy((h @ w[2]).float(), target)
        rows_grad, *grads = torch.autograd.grad(loss, [rows] + w)
        return loss.detach(), [self.embed.grad(rows_grad, tokens, torch.empty_like(self.weights[0]))] + grads

    def step(self, grads, adamw, muon):
        for mine, g in zip(self.grads, grads):
            mine.copy_(g)
        self.all.clip(max_norm=1.0, out=self.record)
        self.muon.step(muon, self.record)
        self.adamw.step(adamw, self.record)


def train(steps=60, quiet=False):
    """Losses of all steps."""
    gen = torch.Generator(device="cuda").manual_seed(0)
    masters = [torch.randn(s, generator=gen, device="cuda") / s[0] ** 0.5 for s in SHAPES]
    masters[0] *= VOCAB ** 0.5 * 0.5
    # text whose next token is mostly a function of the last two
    rule = torch.randint(0, VOCAB, (VOCAB, VOCAB), generator=gen, device="cuda")
    ranks = [Replica(masters) for _ in range(2)]
    adamw = fr.fr_adamw(2e-3, 0.9, 0.99, 1e-8, 0.01, 0)
    muon = fr.muon(lr=2e-2, weight_decay=0.01)
    losses = []
    for step in range(steps):
        parts = []
        for rank in ranks:
            tokens = torch.randint(0, VOCAB, (BATCH, CONTEXT), generator=gen, device="cuda")
            parts.append(rank.differentiate(tokens, rule[tokens[:, -1] // 8, tokens[:, -2] // 8]))
        mean = [(a.float() + b.float()).mul_(0.5).bfloat16() for a, b in zip(parts[0][1], parts[1][1])]
        losses.append(float(parts[0][0] + parts[1][0]) / 2)
        adamw.step = muon.step = step + 1
        for rank in ranks:
            rank.step(mean, adamw, muon)
        if any(rank.muon.sync_status() != fr.FR_OK for rank in ranks):
            raise RuntimeError("a wait was given up in step %d: its replica is to be restored" % step)
        n = fr.diff(ranks[0].plan.fingerprint(), ranks[1].plan.fingerprint())[1]
        if n:
            raise RuntimeError("the replicas differ in %d chunks after step %d" % (n, step))
        if not quiet and step % 10 == 9:
            print("step %3d  loss %.4f  gradient norm %.3f  replicas agree" % (step + 1, losses[-1], fr.clip_view(ranks[0].record)[0]))
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    train(ap.parse_args().steps)
