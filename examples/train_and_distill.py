"""Trains a small language model with the package's steps and losses, distils it into a
smaller one from its top logits, and trains that one on its own samples for a reward.

The model is as small as shows every part in its place: token embedding, one residual
matrix on the embedding of the last token and one on that of the token before,
LM head.  The losses at the head give dX and dW (muon_head_xent, muon_head_distill, the
log probabilities of muon_head_logprob with the gradient of an objective on them); all
gradients are clipped by their global norm (MuonGrads), the two matrices stepped by Muon
(muon_step), embedding and head by AdamW, which clips as it reads (muon_adamw_step), in
fp32 master weights with bf16 copies for the products.  The teacher's entries come from
its logits in one pass (muon_logits_logprob).  The data is a synthetic second-order
Markov chain.

    python examples/train_and_distill.py [--steps 300] [--dim 256] [--vocab 4096]
"""

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))

from paper_2502_16982_b200 import binding as mb  # noqa: E402


class Model:
    """Master weights in fp32, bf16 copies for the products, optimizer state."""

    def __init__(self, vocab, dim, seed, max_norm=float("inf")):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def init(*shape, std):
            return torch.randn(*shape, generator=g, device="cuda") * std

        self.vocab, self.dim = vocab, dim
        self.embed, self.head = init(vocab, dim, std=1.0), init(vocab, dim, std=0.02)
        self.mats = init(2, dim, dim, std=0.5 / dim ** 0.5)
        self.mats16 = self.mats.to(torch.bfloat16)
        self.embed16, self.head16 = self.embed.to(torch.bfloat16), self.head.to(torch.bfloat16)
        self.mats_grad = torch.zeros_like(self.mats)
        self.momentum = torch.zeros_like(self.mats)
        # Muon writes the bf16 copies of its matrices itself
        views = [[t[i] for i in range(2)] for t in (self.mats, self.mats_grad, self.momentum, self.mats16)]
        self.muon = mb.MuonContext([(views[0], views[1], views[2], views[3])])
        self.moments = [torch.zeros_like(t) for t in (self.embed, self.embed, self.head, self.head)]
        self.embed_grad = torch.zeros_like(self.embed)
        self.head_grad = torch.empty_like(self.head16)
        self.max_norm = max_norm
        self.all_grads = mb.MuonGrads([self.mats_grad, self.embed_grad, self.head_grad])
        self.mats_only = mb.MuonGrads([self.mats_grad])
        self.steps = 0

    def hidden(self, tokens):
        """Hidden states of every position from the third on; what backward needs."""
        last, before = tokens[:, 1:-1].reshape(-1), tokens[:, :-2].reshape(-1)
        a, b = self.embed16[last], self.embed16[before]
        x = a + a @ self.mats16[0].t() + b @ self.mats16[1].t()
        return x, (last, before, a, b)

    def backward(self, dx, kept):
        last, before, a, b = kept
        self.mats_grad[0] = dx.t().float() @ a.float()
        self.mats_grad[1] = dx.t().float() @ b.float()
        self.embed_grad.zero_()
        self.embed_grad.index_add_(0, last, (dx + dx @ self.mats16[0]).float())
        self.embed_grad.index_add_(0, before, (dx @ self.mats16[1]).float())

    def step(self, lr):
        self.steps += 1
        total = self.all_grads.muon_grad_norm(self.max_norm)
        self.mats_only.muon_clip_grads(self.max_norm, sum_sq=total.sum_sq)
        self.muon.muon_step(mb.Hyper(lr=lr, wd=0.0), coef=total.coef)
        mb.muon_adamw_step([self.embed, self.head], [self.embed_grad, self.head_grad], self.moments[0::2],
                           self.moments[1::2], self.steps, lr=lr, wd=0.0, coef=total.coef)
        self.embed16.copy_(self.embed)
        self.head16.copy_(self.head)


class Chain:
    """Second-order Markov chain: a token follows from the two before it or, one time in
    eight, at random."""

    def __init__(self, vocab, seed):
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.vocab = vocab
        self.next1 = torch.randint(0, vocab, (vocab,), generator=self.g, device="cuda")
        self.shift = torch.randint(0, 4, (vocab,), generator=self.g, device="cuda")

    def batch(self, rows, length):
        t = torch.randint(0, self.vocab, (rows, length), generator=self.g, device="cuda")
        stray = torch.rand(rows, length, generator=self.g, device="cuda") < 0.125
        for i in range(2, length):
            t[:, i] = torch.where(stray[:, i], t[:, i], self.follow(t[:, i - 1], t[:, i - 2]))
        return t

    def follow(self, last, before):
        return (self.next1[last] + self.shift[before]) % self.vocab


def train(model, chain, steps, lr, rows, length):
    """Next-token training; the first eighth of every row is prompt and carries no loss."""
    losses = []
    for _ in range(steps):
        tokens = chain.batch(rows, length)
        targets = tokens[:, 2:].clone()
        targets[:, : length // 8] = -100
        x, kept = model.hidden(tokens)
        r = mb.muon_head_xent(x, model.head16, targets.reshape(-1), z_loss=1e-4, dx=True, dw=model.head_grad)
        model.backward(r.dx, kept)
        model.step(lr)
        losses.append(r.total)
    return torch.cat(losses).tolist()


def distil(student, teacher, chain, steps, lr, rows, length, top, temperature):
    """The student follows the teacher's `top` largest logits."""
    losses = []
    for _ in range(steps):
        tokens = chain.batch(rows, length)
        best = mb.muon_logits_logprob(teacher.hidden(tokens)[0] @ teacher.head16.t(), top=top, logit_scale=1 / temperature)
        x, kept = student.hidden(tokens)
        r = mb.muon_head_distill(x, student.head16, best.top_ids, best.top_logits, temperature=temperature, teacher_lse=best.lse,
                                 scale=temperature ** 2, dx=True, dw=student.head_grad)
        student.backward(r.dx, kept)
        student.step(lr)
        losses.append(r.total)
    return torch.cat(losses).tolist()


def reinforce(model, chain, steps, lr, rows, length, bonus=1e-3):
    """The model's own next tokens are rewarded where the chain would continue so: one
    policy-gradient step a batch, the mean reward as baseline, with a bonus on the entropy."""
    rewards = []
    for _ in range(steps):
        tokens = chain.batch(rows, length)
        x, kept = model.hidden(tokens)
        with torch.no_grad():
            z = (x @ model.head16.t()).float()
            sampled = torch.multinomial(torch.softmax(z, dim=1), 1, generator=chain.g)[:, 0]
        reward = (sampled == chain.follow(tokens[:, 1:-1], tokens[:, :-2]).reshape(-1)).float()
        r = mb.muon_head_logprob(x, model.head16, sampled)
        n = reward.numel()
        d = mb.muon_head_logprob_grad(x, model.head16, sampled, r, g_logprob=(reward.mean() - reward) / n,
                                      g_entropy=torch.full_like(reward, -bonus / n), dx=True, dw=model.head_grad)
        model.backward(d.dx, kept)
        model.step(lr)
        rewards.append(reward.mean())
    return torch.stack(rewards).tolist() if rewards else []


def perplexity_loss(model, chain, rows, length):
    tokens = chain.batch(rows, length)
    x, _ = model.hidden(tokens)
    return float(mb.muon_head_xent(x, model.head16, tokens[:, 2:].reshape(-1).contiguous()).total)


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--steps", type=int, default=300)
    p.add_argument("--dim", type=int, default=256)
    p.add_argument("--vocab", type=int, default=4096)
    p.add_argument("--rows", type=int, default=64)
    p.add_argument("--length", type=int, default=66)
    p.add_argument("--lr", type=float, default=3e-3)
    p.add_argument("--clip", type=float, default=float("inf"), help="largest global gradient norm")
    p.add_argument("--policy-steps", type=int, default=40)
    a = p.parse_args(argv)
    chain = Chain(a.vocab, 1)
    teacher = Model(a.vocab, a.dim, 2, a.clip)
    first = perplexity_loss(teacher, chain, a.rows, a.length)
    losses = train(teacher, chain, a.steps, a.lr, a.rows, a.length)
    taught = perplexity_loss(teacher, chain, a.rows, a.length)
    print("teacher: loss %.3f -> %.3f over %d steps, held out %.3f -> %.3f" % (losses[0], losses[-1], a.steps, first, taught))
    student = Model(a.vocab, a.dim // 2, 3, a.clip)
    kd = distil(student, teacher, chain, a.steps, a.lr, a.rows, a.length, 32, 2.0)
    final = perplexity_loss(student, chain, a.rows, a.length)
    print("student: distillation loss %.3f -> %.3f over %d steps, held-out loss %.3f" % (kd[0], kd[-1], a.steps, final))
    reward = reinforce(student, chain, a.policy_steps, a.lr / 10, a.rows, a.length)
    if reward:
        print("student on its own samples: reward %.3f -> %.3f over %d steps" % (reward[0], reward[-1], a.policy_steps))
    for m in (teacher, student):
        status, which = m.muon.muon_status()
        assert status == 0, (status, which)
    return {"teacher": losses, "first": first, "taught": taught, "student": kd, "final": final, "reward": reward}


if __name__ == "__main__":
    main()
