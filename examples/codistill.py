"""Workers that learn from each other's answers: mixtures of experts trained by distillation from a neighbour's top logits.

Every one of the k workers (k sets of buffers on one GPU) has a mixture of its own and its own tokens with labels; the neighbour on a ring has answered the same
tokens, and what it sends are the top logits of each answer and their places, a few numbers a token, where gradients would be a model's size.
A step, for all workers in each call:

  1. router logits = x @ router; experts and weights of every token (bagua_route), the balance loss of all tokens and its gradient (bagua_balance_stats,
     bagua_balance_grad);
  2. answer = sum of weight * (x @ expert) over a token's experts, logits over the vocabulary;
  3. loss and gradient of the answers by the neighbour's top logits and the labels (bagua_distill_loss, bagua_distill_grad, in place);
  4. back through the mixture: experts, and the router through the weights (bagua_route_grad);
  5. each worker's gradient norm with its clipping factor, and AdamW (bagua_grad_norm, bagua_adamw_step).

  python examples/codistill.py [--workers 4] [--steps N]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2107_01499_amd as bg  # noqa: E402


def empty(shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype, device="cuda")


class Mixtures:
    """k workers' mixtures, and the buffers of a step."""

    def __init__(self, workers=4, tokens=256, width=32, experts=8, top_k=2, vocab=200, sent=16, temperature=2.0, label_weight=0.5, alpha=0.01, seed=0):
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.workers, self.tokens, self.width, self.experts, self.top_k, self.vocab, self.sent = workers, tokens, width, experts, top_k, vocab, sent
        self.temperature, self.label_weight, self.alpha = temperature, label_weight, alpha
        w, t = range(workers), tokens
        self.router = [torch.randn(width, experts, device="cuda", generator=self.g) / width ** 0.5 for _ in w]
        self.expert = [torch.randn(width, experts * vocab, device="cuda", generator=self.g) / width ** 0.5 for _ in w]
        self.drouter, self.dexpert = [torch.zeros_like(p) for p in self.router], [torch.zeros_like(p) for p in self.expert]
        self.ids, self.weights, self.dweights = [empty((t, top_k), torch.int64) for _ in w], [empty((t, top_k)) for _ in w], [empty((t, top_k)) for _ in w]
        self.dchoice, self.dbalance = [empty((t, experts)) for _ in w], [empty((t, experts)) for _ in w]
        self.counts, self.prob, self.balance, self.load = empty(experts + 1, torch.int32), empty(experts), empty(1), empty(experts)
        self.ws = empty(bg.bagua_balance_workspace_bytes(experts), torch.uint8)
        self.loss, self.stats = [empty(t) for _ in w], [empty((t, 3)) for _ in w]
        self.distill_ws = empty(bg.bagua_distill_workspace_bytes(workers * t, vocab), torch.uint8)
        self.per_token = torch.full((1,), 1.0 / t, device="cuda")                   # the loss of a worker is the mean over its tokens
        # what the labels follow: a map that no worker has
        self.truth = torch.randn(width, vocab, device="cuda", generator=self.g) * 3 / width ** 0.5

    def batch(self):
        """Each worker's tokens, their labels (some unknown), and which of them are no padding."""
        xs = list(torch.randn(self.workers, self.tokens, self.width, device="cuda", generator=self.g).unbind())
        labels = [torch.where(torch.rand(self.tokens, device="cuda", generator=self.g) < 0.1, -100, (x @ self.truth).argmax(1)) for x in xs]
        mask = [torch.rand(self.tokens, device="cuda", generator=self.g) >= 0.1 for _ in xs]
        return xs, labels, mask

    def answers(self, xs, owner, mask):
        """Answers of worker owner(i)'s mixture to the tokens of worker i, and what the way back needs."""
        z = [x @ self.router[owner(i)] for i, x in enumerate(xs)]
        bg.bagua_route(z, mask, self.ids, self.weights)
        outs, logits = [], []
        for i, x in enumerate(xs):
            out = (x @ self.expert[owner(i)]).view(self.tokens, self.experts, self.vocab)
            chosen = out.gather(1, self.ids[i].clamp(min=0)[:, :, None].expand(-1, -1, self.vocab))      # (a padded token's weights are 0)
            outs.append(chosen)
            logits.append((chosen * self.weights[i][:, :, None]).sum(1))
        return z, outs, logits

    def sent_by_neighbours(self, xs, mask):
        """The top logits of the answers of each worker's neighbour, and their places."""
        _, _, logits = self.answers(xs, lambda i: (i + 1) % self.workers, mask)
        top = [torch.topk(a, self.sent, dim=1) for a in logits]
        return [t.values for t in top], [t.indices for t in top]

    def gradients(self, xs, labels, mask, teacher, places):
        """Fills drouter and dexpert; returns the workers' losses."""
        z, outs, logits = self.answers(xs, lambda i: i, mask)
        bg.bagua_balance_stats(z, self.ids, mask, self.counts, self.prob, self.ws, self.alpha, self.balance, self.load)
        bg.bagua_balance_grad(z, mask, self.load, None, self.dbalance)
        bg.bagua_distill_loss(logits, places, teacher, labels, mask, self.loss, self.stats, self.distill_ws, self.temperature, 1.0, self.label_weight)
        bg.bagua_distill_grad(logits, places, teacher, labels, mask, self.stats, self.per_token, logits, self.temperature, 1.0, self.label_weight)
        for d, out, dw in zip(logits, outs, self.dweights):
            torch.sum(out * d[:, None, :], 2, out=dw)
        bg.bagua_route_grad(None, self.ids, self.weights, self.dweights, self.dchoice)
        for i, x in enumerate(xs):
            d = empty((self.tokens, self.experts, self.vocab))
            d.scatter_(1, self.ids[i].clamp(min=0)[:, :, None].expand(-1, -1, self.vocab), self.weights[i][:, :, None] * logits[i][:, None, :])
            torch.mm(x.t(), d.view(self.tokens, -1), out=self.dexpert[i])
            torch.mm(x.t(), self.dchoice[i] + self.dbalance[i], out=self.drouter[i])
        return [l.mean() for l in self.loss]


def train(steps=100, workers=4, lr=3e-3, seed=0, tell=None, **more):
    """Returns the mean loss of every step."""
    m = Mixtures(workers, seed=seed, **more)
    plans, clips = [], [empty(2) for _ in range(workers)]
    for i in range(workers):
        params, grads = [m.router[i], m.expert[i]], [m.drouter[i], m.dexpert[i]]
        ws = empty(bg.bagua_tensor_plan_bytes([p.numel() for p in params]), torch.uint8)
        plans.append(bg.bagua_tensor_plan(grads, ws, params=params, m=[torch.zeros_like(p) for p in params], v=[torch.zeros_like(p) for p in params]))
    history = []
    for step in range(1, steps + 1):
        xs, labels, mask = m.batch()
        losses = m.gradients(xs, labels, mask, *m.sent_by_neighbours(xs, mask))
        for plan, clip in zip(plans, clips):
            bg.bagua_grad_norm(plan, clip, 1.0)
            bg.bagua_adamw_step(plan, step, lr, clip=clip, seed=step)
        history.append(torch.stack(losses).mean())
        if tell and step % 10 == 0:
            tell("step %4d   loss %.4f   balance %.4f" % (step, float(history[-1]), float(m.balance) / m.alpha))
    return torch.stack(history).tolist()


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--workers", type=int, default=4)
    a = ap.parse_args()
    train(a.steps, a.workers, tell=lambda s: print(s, flush=True))
