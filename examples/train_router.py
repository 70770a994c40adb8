"""Data-parallel training of a mixture's router, with the balance loss of the whole batch, compressed gradients and AdamW.

Every one of the k workers (k sets of buffers on one GPU) has its own tokens.  A step:

  1. logits = tokens @ weight + bias, the top-k experts of each token; the task wants every token at the expert of its kind, and some
     kinds are far more frequent than others, so that the task alone overloads a few experts;
  2. balance loss of all workers' tokens together and its gradient (bagua_balance_stats, bagua_balance_grad), added to the task's;
  3. each worker's gradients of weight and bias are flattened into its bucket and compressed with error feedback
     (bagua_bucket_flatten_run, bagua_compress_minmax_u8), averaged and compressed again by the server step
     (bagua_decompress_reduce_recompress);
  4. norm and clipping factor of the averaged gradients, AdamW on weight and bias (bagua_grad_norm, bagua_adamw_step).

  python examples/train_router.py [--alpha 0] [--state-bits 32] [--steps N]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2107_01499_amd as bg  # noqa: E402

CHUNK = 1024


def empty(shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype, device="cuda")


class Workers:
    """k workers' tokens, and the buffers that their gradients go through."""

    def __init__(self, workers, tokens, width, experts, generator):
        self.g, self.width, self.experts = generator, width, experts
        self.kinds = torch.randn(experts, width, device="cuda", generator=generator)
        self.frequency = 1.0 / torch.arange(1, experts + 1, device="cuda")            # of the kinds: the first ones make up most tokens
        self.tokens, self.workers = tokens, workers
        # a worker's gradients, and the bucket they are flattened into
        self.grads = [[empty((width, experts)), empty(experts)] for _ in range(workers)]
        n = self.n = width * experts + experts
        nc = bg.num_chunks(n, CHUNK)
        self.plans = []
        for grads in self.grads:
            ws = empty(bg.bagua_flatten_workspace_bytes(2, n), torch.uint8)
            bg.bagua_flatten_plan(grads, [0, width * experts], n, ws)
            self.plans.append(ws)
        self.bucket, self.left_out = empty(n), [empty(n) for _ in range(workers)]
        self.codes, self.ranges = [empty(n, torch.uint8) for _ in range(workers)], [empty(2 * nc) for _ in range(workers)]
        self.server_left_out, self.codes_back, self.ranges_back = empty(n), empty(n, torch.uint8), empty(2 * nc)
        self.average = empty(n)

    def batch(self):
        """Each worker's tokens, and their kinds."""
        kind = torch.multinomial(self.frequency.expand(self.workers, -1), self.tokens, replacement=True, generator=self.g)
        noise = 3.0 * torch.randn(self.workers, self.tokens, self.width, device="cuda", generator=self.g)
        return list((self.kinds[kind] + noise).unbind()), list(kind.unbind())

    def exchange(self):
        """The average of the workers' gradients, as every worker has it after one C_LP_S round."""
        for i in range(self.workers):
            bg.bagua_bucket_flatten_run(self.plans[i], 2, self.bucket)
            bg.bagua_compress_minmax_u8(self.bucket, self.left_out[i], CHUNK, self.codes[i], self.ranges[i])
        bg.bagua_decompress_reduce_recompress(bg.CODEC_MINMAX_U8, self.codes, self.ranges, self.server_left_out, self.n, CHUNK, self.codes_back,
                                              self.ranges_back, self.average)


def train(steps=150, workers=4, tokens=2048, width=128, experts=16, top_k=2, alpha=0.5, state_bits=8, lr=1e-2, seed=0, tell=None):
    """Returns, for every step, (balance loss before alpha, share of the most popular expert times the number of experts, gradient norm)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = Workers(workers, tokens, width, experts, g)
    params = [torch.randn(width, experts, device="cuda", generator=g) / width ** 0.5, empty(experts)]
    # the optimizer works on the averaged bucket's two tensors
    grads = [w.average[:width * experts].view(width, experts), w.average[width * experts:]]
    state = torch.float32 if state_bits == 32 else torch.float8_e4m3fn
    m, v = ([torch.zeros(p.shape, device="cuda").to(state) for p in params] for _ in range(2))
    scales = {}
    if state_bits == 8:
        scales = {k: [empty((p.numel() + 255) // 256) for p in params] for k in ("m_scales", "v_scales")}
    plan = bg.bagua_tensor_plan(grads, empty(bg.bagua_tensor_plan_bytes([p.numel() for p in params]), torch.uint8), params=params, m=m, v=v,
                                decay=[1.0, 0.0], **scales)
    clip = empty(2)
    counts, prob, loss, weight = empty(experts + 1, torch.int32), empty(experts), empty(1), empty(experts)
    ws = empty(bg.bagua_balance_workspace_bytes(experts), torch.uint8)
    # the balance loss is of all workers' tokens: a worker's share of it is as large as the average over workers makes it small
    upstream = torch.full((1,), alpha * workers, device="cuda")
    history = []
    for step in range(1, steps + 1):
        xs, kinds = w.batch()
        logits = [x @ params[0] + params[1] for x in xs]
        ids = [torch.topk(z, top_k, dim=1).indices for z in logits]
        bg.bagua_balance_stats(logits, ids, None, counts, prob, ws, 1.0, loss, weight)
        dbalance = [torch.empty_like(z) for z in logits]
        bg.bagua_balance_grad(logits, None, weight, upstream, dbalance)
        for x, z, kind, d, (dw, db) in zip(xs, logits, kinds, dbalance, w.grads):
            task = torch.softmax(z, 1)
            task[torch.arange(tokens, device="cuda"), kind] -= 1.0
            d = task / tokens + d
            torch.mm(x.t(), d, out=dw)
            torch.sum(d, 0, out=db)
        w.exchange()
        bg.bagua_grad_norm(plan, clip, 1.0)
        bg.bagua_adamw_step(plan, step, lr, weight_decay=0.01, clip=clip, seed=step)
        load = counts[:experts].float()
        history.append(torch.stack([loss[0], load.max() / load.sum() * experts, clip[0]]))
        if tell and step % 10 == 0:
            tell("step %4d   balance %.4f   most popular expert %.2f times its share   gradient norm %.3f" % (step, *history[-1].tolist()))
    return torch.stack(history).tolist()


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=150)
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--experts", type=int, default=16)
    ap.add_argument("--alpha", type=float, default=0.5)
    ap.add_argument("--state-bits", type=int, choices=(8, 32), default=8)
    a = ap.parse_args()
    train(a.steps, a.workers, experts=a.experts, alpha=a.alpha, state_bits=a.state_bits, tell=lambda s: print(s, flush=True))
