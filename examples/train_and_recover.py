"""Train with data-parallel replicas, lose one, restore it from another and train on.

Two replicas of a small network on one GPU, each with its own bf16 weights, fp32 masters and Adam moments (32 or 8 bits).
Every step each replica differentiates its half of the batch, the gradients are averaged, and each replica clips them and
makes its AdamW step by itself.  The step gives the same bits on both, so their fingerprints agree chunk for chunk (Sec.
III-A of FlashRecovery, arXiv 2509.03047: replicas hold the same states).  Then one replica fails in its optimizer step: the
step tags say that training resumes with the following step (Sec. III-E), its state is restored from the other replica's
memory, and both go on.

    python examples/train_and_recover.py [--bits 8] [--steps 40] [--fail-at 20]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2509_03047_gb300 import flashrec as fr  # noqa: E402
from paper_2509_03047_gb300 import steptag  # noqa: E402

SHAPES = [(64, 512), (512,), (512, 512), (512,), (512, 10)]  # two hidden layers
CHUNK = 64 << 10


class Replica:
    """One rank: its state, the plan of its optimizer step and the plan by which it is fingerprinted and restored."""

    def __init__(self, masters, bits):
        dev = masters[0].device
        self.masters = [x.clone() for x in masters]
        self.weights = [x.bfloat16() for x in masters]
        self.grads = [torch.zeros_like(x) for x in self.weights]
        if bits == 8:
            self.m, self.v = ([torch.zeros(x.numel(), dtype=torch.uint8, device=dev) for x in masters] for _ in range(2))
            blocks = [-(-x.numel() // fr.FR_OPT_BLOCK) for x in masters]
            self.exps = [[torch.zeros(k, dtype=torch.uint8, device=dev) for k in blocks] for _ in range(2)]
        else:
            self.m, self.v = ([torch.zeros_like(x) for x in masters] for _ in range(2))
            self.exps = [None, None]
        # biases do not decay
        self.opt = fr.OptPlan(self.weights, self.grads, self.m, self.v, masters=self.masters, m_exp=self.exps[0],
                              v_exp=self.exps[1], decay_scale=[float(x.dim() > 1) for x in masters])
        self.record = self.opt.new_clip()
        self.state = [t for group in (self.weights, self.masters, self.m, self.v, *self.exps) if group for t in group]
        self.plan = fr.Plan(self.state, CHUNK)

    def differentiate(self, x, y):
        """(loss, gradients) of this replica's part of the batch, by its own weights."""
        w = [t.detach().requires_grad_() for t in self.weights]
        h = torch.relu(x @ w[0] + w[1])
        h = torch.relu(h @ w[2] + w[3])
        loss = torch.nn.functional.cross_entropy((h @ w[4]).float(), y)
        return loss.detach(), torch.autograd.grad(loss, w)

    def step(self, grads, hyper):
        for mine, g in zip(self.grads, grads):
            mine.copy_(g)
        self.opt.clip(max_norm=1.0, out=self.record)  # stays on the device: the step reads it there
        self.opt.step(hyper, self.record)


def differing_chunks(a, b):
    return fr.diff(a.plan.fingerprint(), b.plan.fingerprint())[1]


def restore(failed, source):
    """`failed`'s state from `source`'s memory, checked chunk by chunk on the way; chunks that do not verify are sent again."""
    staging, count = source.plan.new_packed(), torch.empty(1, dtype=torch.int64, device="cuda")
    ta, tb = source.plan.new_table(), failed.plan.new_table()
    fr.fr_restore_fp(source.plan.handle, failed.plan.handle, staging, 2, None, count, ta, tb)
    if int(count) or fr.diff(ta, tb)[1]:
        raise RuntimeError("the restored state differs from its source")


def train(bits=8, steps=40, fail_at=20, quiet=False):
    """Losses of all steps."""
    gen = torch.Generator(device="cuda").manual_seed(0)
    masters = [torch.randn(s, generator=gen, device="cuda") / (s[0] ** 0.5 if len(s) > 1 else 1e9) for s in SHAPES]
    data = torch.randn(4096, 64, generator=gen, device="cuda")
    labels = (data @ torch.randn(64, 10, generator=gen, device="cuda")).argmax(1)
    ranks = [Replica(masters, bits) for _ in range(2)]
    controller = steptag.Controller(2, [[0, 1]])
    hyper = fr.fr_adamw(2e-3, 0.9, 0.99, 1e-8, 0.01, 0, 1234, fr.FR_ROUND_RANDOM)
    losses, step = [], 0
    while step < steps:
        for r in range(2):
            controller.heartbeat(r, step)
        rows = torch.randint(0, 4096, (512,), generator=gen, device="cuda")
        parts = [rank.differentiate(data[rows[r::2]].bfloat16(), labels[rows[r::2]]) for r, rank in enumerate(ranks)]
        mean = [(a.float() + b.float()).mul_(0.5).bfloat16() for a, b in zip(parts[0][1], parts[1][1])]
        losses.append(float(parts[0][0] + parts[1][0]) / 2)
        hyper.step = step + 1
        if step == fail_at:  # rank 1 is lost in its optimizer step, rank 0 finishes its own
            controller.heartbeat(1, steptag.OPTIMIZER)
            ranks[0].step(mean, hyper)
            controller.heartbeat(0, step + 1)
            for t in ranks[1].state:
                t.view(torch.uint8).fill_(0xA5)
            controller.report_failure(1)
            decision = controller.decide()
            restore(ranks[1], ranks[decision.source[1]])
            controller.failed.clear()
            step = decision.resume_step
            if not quiet:
                print("rank 1 lost in the optimizer step of step %d, restored; resuming at step %d" % (fail_at, step))
        else:
            for rank in ranks:
                rank.step(mean, hyper)
            step += 1
        n = differing_chunks(*ranks)
        if n:
            raise RuntimeError("the replicas differ in %d chunks after step %d" % (n, step))
        if not quiet and step % 10 == 0:
            norm, scale, bad = fr.clip_view(ranks[0].record)
            print("step %3d  loss %.4f  gradient norm %.3f  factor %.3f  replicas agree" % (step, losses[-1], norm, scale))
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--bits", type=int, choices=(8, 32), default=8)
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--fail-at", type=int, default=20)
    a = ap.parse_args()
    train(a.bits, a.steps, a.fail_at)
