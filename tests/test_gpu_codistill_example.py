"""Workers that learn from each other's answers (examples/codistill.py): routing, balance loss, distillation, norm and AdamW together."""
import importlib.util
import math
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def example():
    assert torch.cuda.is_available()
    spec = importlib.util.spec_from_file_location("codistill", os.path.join(ROOT, "examples", "codistill.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_it_runs(example):
    history = example.train(steps=5, workers=3, tokens=65, vocab=101, experts=6, top_k=3)
    assert len(history) == 5 and all(math.isfinite(h) for h in history)
    assert history == example.train(steps=5, workers=3, tokens=65, vocab=101, experts=6, top_k=3)      # the same seed gives the same run


@pytest.mark.parametrize("experts,top_k", [(8, 2), (6, 1), (70, 3)])
def test_a_step_has_the_gradients_of_its_loss(example, experts, top_k):
    """All of a step's gradients against automatic differentiation of the same loss in 64 bits."""
    m = example.Mixtures(workers=3, tokens=65, width=16, experts=experts, top_k=top_k, vocab=101, sent=7)
    xs, labels, mask = m.batch()
    teacher, places = m.sent_by_neighbours(xs, mask)
    m.gradients(xs, labels, mask, teacher, places)
    router, expert = ([p.double().clone().requires_grad_() for p in ps] for ps in (m.router, m.expert))
    total = torch.zeros((), dtype=torch.float64, device="cuda")
    probability, chosen, tokens = torch.zeros(experts, dtype=torch.float64, device="cuda"), torch.zeros(experts, dtype=torch.float64, device="cuda"), 0
    for i, x in enumerate(xs):
        x, ids, keep = x.double(), m.ids[i].clamp(min=0), mask[i]
        z = x @ router[i]
        assert torch.equal(torch.topk(z, top_k, dim=1).indices[keep], ids[keep])
        w = torch.softmax(z.gather(1, ids), 1) * keep[:, None]
        out = (x @ expert[i]).view(65, experts, 101).gather(1, ids[:, :, None].expand(-1, -1, 101))
        answer = (out * w[:, :, None]).sum(1)
        t = m.temperature
        log_q, log_p = torch.log_softmax(teacher[i].double() / t, 1), torch.log_softmax(answer / t, 1).gather(1, places[i])
        loss = t * t * (log_q.exp() * (log_q - log_p)).sum(1)
        cross = -torch.log_softmax(answer, 1).gather(1, labels[i].clamp(min=0)[:, None])[:, 0]
        total = total + ((loss + m.label_weight * cross * (labels[i] >= 0)) * keep).mean()
        probability = probability + (torch.softmax(z, 1) * keep[:, None]).sum(0)
        chosen += torch.bincount(ids[keep].view(-1), minlength=experts)
        tokens += int(keep.sum())
    total = total + m.alpha * experts * (chosen / (top_k * tokens) * probability / tokens).sum()
    total.backward()
    for got, want in zip(m.drouter + m.dexpert, router + expert):
        # an element is a sum over 65 tokens of products; x, the answers (sums of 16 products, up to 10) and the softmax of these are off by some 40 U of what
        # they are made of, and what is added up is at most of the size of the largest gradient times the tokens
        assert torch.all((got.double() - want.grad).abs() <= 65 * 100 * U * want.grad.abs().max())
