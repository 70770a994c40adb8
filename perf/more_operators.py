"""Operators on rows of logits whose speed is looked after: the routing of tokens to experts, which gives the balance loss its choices,
and distillation from a teacher's top logits, with which workers learn from each other's answers instead of each other's gradients.

A case is one call of one operator ("kind"):

  route         of every token the top-k experts and their weights.  score "softmax" or "sigmoid"; with bias, experts are chosen by score +
                bias and weighted by the score alone; groups > 1: only experts of the best `top_groups` groups are chosen, a group being as good as the
                sum of its `group_best` best experts; renormalised: a token's weights are divided by their sum.
  route_grad    its backward: gradient of the router's logits from that of the weights.
  distill       of every row the divergence of the student's softmax from the teacher's, which is the softmax of its top logits alone, both
                at a temperature, and the cross entropy of a label, each with a factor; and what the backward pass needs of the row.
  distill_grad  its backward: gradient of the student's logits.

Where `own` is false the operators are computed in plain torch operations in 32 bits; what experts are chosen by is computed in 64, since
scores lie next to each other.  Ties go to the lowest index.
"""
import math

import torch

own = False

LARGEST = 2.16e9             # bytes: no drawn case needs more than the largest listed one
SOFTMAX, SIGMOID = "softmax", "sigmoid"
UP = 1.0 / 1024.0            # the gradient that arrives at a row's loss: that of a mean


def _route(name, workers, tokens, experts, top, dtype, score=SOFTMAX, biased=False, groups=1, top_groups=1, group_best=1, renormalise=True, scale=1.0,
           masked=False, ids="i64"):
    return dict(name=name, kind="route", workers=workers, tokens=tokens, experts=experts, top=top, dtype=dtype, score=score, biased=biased, groups=groups,
                top_groups=top_groups, group_best=group_best, renormalise=renormalise, scale=scale, masked=masked, ids=ids)


def _route_grad(name, workers, tokens, experts, top, dtype, score=SOFTMAX, renormalise=True, scale=1.0, masked=False, ids="i64"):
    return dict(name=name, kind="route_grad", workers=workers, tokens=tokens, experts=experts, top=top, dtype=dtype, score=score,
                renormalise=renormalise, scale=scale, masked=masked, ids=ids)


def _distill(name, kind, workers, rows, vocab, top, dtype, temperature=1.0, label=0.0, masked=False):
    return dict(name=name, kind=kind, workers=workers, rows=rows, vocab=vocab, top=top, dtype=dtype, temperature=temperature, label=label, masked=masked)


def listed():
    return [
        # a few sequences' next tokens through a small mixture: the call itself counts
        _route("route_small", 1, 96, 8, 2, "f32"),
        # eight workers' padded batches through 64 experts
        _route("route_8_workers", 8, 32768, 64, 6, "bf16", masked=True),
        # a long batch, experts chosen with a bias for balance out of half of the groups
        _route("route_groups", 1, 131072, 256, 8, "f32", SIGMOID, biased=True, groups=8, top_groups=4, group_best=2, scale=2.5),
        # probabilities of the whole row with a bias, an odd number of experts
        _route("route_bias_odd", 2, 16411, 60, 4, "bf16", biased=True, renormalise=False, ids="i32"),
        # four workers, an odd number of experts, independent scores
        _route_grad("route_grad_odd", 4, 4099, 60, 4, "f32", SIGMOID, masked=True),
        # a long batch through many experts
        _route_grad("route_grad_large", 1, 262144, 256, 8, "bf16"),
        # one short sequence over a small vocabulary
        _distill("distill_small", "distill", 1, 24, 1009, 8, "f32"),
        # few rows over a large vocabulary: a long axis, and hardly a row for every compute unit
        _distill("distill_few_rows", "distill", 1, 40, 200003, 100, "bf16", 2.0, 0.5),
        # eight workers learn from each other's top logits, BERT's vocabulary
        _distill("distill_8_workers", "distill", 8, 512, 30522, 64, "bf16", 2.0, 0.5, masked=True),
        # one short sequence, backward
        _distill("distill_grad_small", "distill_grad", 1, 24, 1009, 8, "f32", 1.0, 0.0),
        # eight workers, backward
        _distill("distill_grad_8_workers", "distill_grad", 8, 512, 30522, 64, "bf16", 2.0, 0.5, masked=True),
        # a batch over a large vocabulary; the largest
        _distill("distill_grad_large", "distill_grad", 1, 4096, 131072, 32, "bf16", 1.0, 0.0),
    ]


def _log(rng, low, high):
    """A whole number, spread over its logarithm; odd ones as often as not."""
    n = int(round(2.0 ** rng.uniform(math.log2(low), math.log2(high))))
    return min(high, n | rng.choice([0, 1]))


def draw(rng):
    """One more case of the same ranges: any kind, sizes spread over their logarithm, odd ones among them."""
    while True:
        kind = rng.choice(["route", "route", "route_grad", "distill", "distill_grad"])
        dtype, masked, workers = rng.choice(["f32", "bf16", "bf16", "f16"]), rng.random() < 0.5, rng.choice([1, 1, 2, 3, 4, 8])
        if kind in ("route", "route_grad"):
            experts = rng.choice([2, 4, 7, 8, 16, 32, 60, 64, 72, 100, 128, 160, 256, 384, 512])
            case = dict(kind=kind, workers=workers, tokens=_log(rng, 1, 1 << 18), experts=experts, top=min(experts, rng.choice([1, 2, 2, 4, 6, 8])), dtype=dtype,
                        score=rng.choice([SOFTMAX, SIGMOID]), renormalise=rng.random() < 0.7, scale=rng.choice([1.0, 2.5]), masked=masked,
                        ids=rng.choice(["i64", "i32"]))
            if kind == "route":
                groups = rng.choice([1, 1, 2, 4, 8])
                if experts % groups or experts // groups < 2:
                    groups = 1
                top_groups = rng.choice([t for t in (1, 2, 3, 4, 8) if t <= groups and t * (experts // groups) >= case["top"]] or [groups])
                case.update(biased=rng.random() < 0.5, groups=groups, top_groups=top_groups, group_best=rng.choice([1, 2]) if groups > 1 else 1)
            if case["tokens"] * workers * experts > 1 << 26:
                continue
        else:
            vocab = _log(rng, 128, 262144)
            case = dict(kind=kind, workers=workers, rows=_log(rng, 1, 1 << 13), vocab=vocab, top=min(vocab, rng.choice([1, 4, 8, 20, 32, 64, 100, 128, 256])),
                        dtype=dtype, temperature=rng.choice([1.0, 2.0, 3.5]), label=rng.choice([0.0, 0.5]), masked=masked)
            if case["rows"] * workers * vocab > 1 << 29:
                continue
        if work(case)["bytes"] <= LARGEST:
            return case


# ---------------------------------------------------------------------------------------------- inputs
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
IDS = {"i32": torch.int32, "i64": torch.int64}


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(shape, g, sigma=1.0):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, sigma, generator=g)


def _rand(shape, g):
    return torch.rand(shape, device="cuda", generator=g)


def _counted_rows(rows, masked):
    """How many of a worker's rows are no padding."""
    return rows - rows // 8 if masked else rows


def _mask(rows, g):
    """Padding at the ends of sequences."""
    order = _rand(max(1, rows // 64 + 1), g).repeat_interleave(64)[:rows].argsort(stable=True)
    mask = torch.zeros(rows, dtype=torch.bool, device="cuda")
    mask[order[:_counted_rows(rows, True)]] = True
    return mask


def prepare(case, seed):
    g = _gen(seed)
    return {"route": _prepare_route, "route_grad": _prepare_route_grad, "distill": _prepare_distill, "distill_grad": _prepare_distill}[case["kind"]](case, g)


def _router_logits(case, g):
    e = case["experts"]
    liking = _normal(e, g, 0.7)                        # some experts are more popular than others
    return [(_normal((case["tokens"], e), g, 1.5) + liking).to(TYPES[case["dtype"]]) for _ in range(case["workers"])]


def _prepare_route(case, g):
    s = dict(case, logits=_router_logits(case, g))
    t, k, w = case["tokens"], case["top"], range(case["workers"])
    s["mask"] = [_mask(t, g) for _ in w] if case["masked"] else None
    s["bias"] = _normal(case["experts"], g, 0.1 if case["score"] == SIGMOID else 0.01) if case["biased"] else None
    s["ids"] = [torch.zeros((t, k), dtype=IDS[case["ids"]], device="cuda") for _ in w]
    s["weights"] = [torch.zeros((t, k), device="cuda") for _ in w]
    return s


def _prepare_route_grad(case, g):
    """What the forward pass has left, and the gradients that arrive at the weights."""
    s = dict(case, logits=_router_logits(case, g), ids=[], weights=[], up=[], out=[])
    t, k = case["tokens"], case["top"]
    for x in s["logits"]:
        ids = torch.topk(x.float(), k, dim=1).indices
        v = torch.gather(x.float(), 1, ids)
        v = torch.exp(v - v.amax(1, keepdim=True)) if case["score"] == SOFTMAX else 1.0 / (1.0 + torch.exp(-v))
        if case["renormalise"]:
            v = v / v.sum(1, keepdim=True)
        elif case["score"] == SOFTMAX:
            v = v / torch.exp(x.float() - x.float().amax(1, keepdim=True)).sum(1, keepdim=True)
        v = v * case["scale"]
        if case["masked"]:
            mask = _mask(t, g)[:, None]
            ids, v = torch.where(mask, ids, torch.full_like(ids, -1)), torch.where(mask, v, torch.zeros_like(v))
        s["ids"].append(ids.to(IDS[case["ids"]]))
        s["weights"].append(v)
        s["up"].append(_normal((t, k), g))
        s["out"].append(torch.zeros_like(x))
    return s


def _prepare_distill(case, g):
    r, v, k, dtype = case["rows"], case["vocab"], case["top"], TYPES[case["dtype"]]
    s = dict(case, logits=[], ids=[], teacher=[], labels=[], mask=[] if case["masked"] else None)
    for _ in range(case["workers"]):
        x = torch.empty((r, v), dtype=dtype, device="cuda").normal_(0.0, 2.0, generator=g)
        # the teacher's top logits, the largest first: of every k-th part of the vocabulary one
        ids = _rand((r, k), g).argsort(1) * (v // k) + (_rand((r, k), g) * (v // k)).long().clamp_(max=v // k - 1)
        top = torch.sort(8.0 - torch.empty((r, k), device="cuda").exponential_(0.4, generator=g), dim=1, descending=True).values
        x.scatter_(1, ids, (0.7 * top + _normal((r, k), g, 1.5)).to(dtype))          # the student has learnt something of it
        s["logits"].append(x)
        s["ids"].append(ids)
        s["teacher"].append(top.to(dtype))
        labels = torch.where(_rand(r, g) < 0.6, ids[:, 0], (_rand(r, g) * v).long().clamp_(max=v - 1))
        s["labels"].append(torch.where(_rand(r, g) < 0.05, torch.full_like(labels, -100), labels))
        if case["masked"]:
            s["mask"].append(_mask(r, g))
    if case["label"] == 0.0:
        s["labels"] = None
    s["loss"] = [torch.zeros(r, device="cuda") for _ in s["logits"]]
    if case["kind"] == "distill_grad":
        # what the forward pass has left: the row's largest logit, the sum of exp((x - largest) / temperature) and, for labels, that of exp(x - largest)
        s["stats"] = [_statistics(x, case["temperature"], case["label"] != 0.0) for x in s["logits"]]
        s["up"] = torch.full((1,), UP, device="cuda")
        s["out"] = [torch.zeros_like(x) for x in s["logits"]]
    else:
        s["stats"] = [torch.zeros((r, 3), device="cuda") for _ in s["logits"]]
        if own:
            import paper_2107_01499_amd as bg
            s["ws"] = torch.empty(bg.bagua_distill_workspace_bytes(case["workers"] * r, v), dtype=torch.uint8, device="cuda")
    return s


def _statistics(x, temperature, labels):
    out = []
    for c in x.split(max(1, (1 << 27) // x.shape[1])):
        c = c.float()
        m = c.amax(1, keepdim=True)
        sum_1 = torch.exp(c - m).sum(1, keepdim=True) if labels else torch.zeros_like(m)
        out.append(torch.cat([m, torch.exp((c - m) / temperature).sum(1, keepdim=True), sum_1], 1))
    return torch.cat(out)


# ---------------------------------------------------------------------------------------------- one call
def run(state):
    if own:
        return _OWN[state["kind"]](state)
    return _PLAIN[state["kind"]](state)


def _score(s, bg):
    return bg.SCORE_SOFTMAX if s["score"] == SOFTMAX else bg.SCORE_SIGMOID


def _own_route(s):
    import paper_2107_01499_amd as bg
    bg.bagua_route(s["logits"], s["mask"], s["ids"], s["weights"], s["bias"], _score(s, bg), s["groups"], s["top_groups"], s["group_best"], s["renormalise"],
                   s["scale"])
    return {"ids": s["ids"], "weights": s["weights"]}


def _own_route_grad(s):
    import paper_2107_01499_amd as bg
    bg.bagua_route_grad(s["logits"], s["ids"], s["weights"], s["up"], s["out"], _score(s, bg), s["renormalise"], s["scale"])
    return s["out"]


def _own_distill(s):
    import paper_2107_01499_amd as bg
    bg.bagua_distill_loss(s["logits"], s["ids"], s["teacher"], s["labels"], s["mask"], s["loss"], s["stats"], s["ws"], s["temperature"], 1.0, s["label"])
    return {"loss": s["loss"], "stats": s["stats"]}


def _own_distill_grad(s):
    import paper_2107_01499_amd as bg
    bg.bagua_distill_grad(s["logits"], s["ids"], s["teacher"], s["labels"], s["mask"], s["stats"], s["up"], s["out"], s["temperature"], 1.0, s["label"])
    return s["out"]


_OWN = {"route": _own_route, "route_grad": _own_route_grad, "distill": _own_distill, "distill_grad": _own_distill_grad}


# ---------------------------------------------------------------------------------------------- plain forms
def _scores(x, score):
    if score == SIGMOID:
        return 1.0 / (1.0 + torch.exp(-x))
    x = torch.exp(x - x.amax(1, keepdim=True))
    return x / x.sum(1, keepdim=True)


def _plain_route(s):
    ids_out, weights_out = [], []
    for i, x in enumerate(s["logits"]):
        by_logit = s["bias"] is None and s["group_best"] == 1                  # scores rise with the logits
        choice = x.float() if by_logit else _scores(x.double(), s["score"])
        if s["bias"] is not None:
            choice = choice + s["bias"].double()
        if s["groups"] > 1:
            t, e = choice.shape
            good = torch.sort(choice.view(t, s["groups"], -1), dim=2, descending=True).values[:, :, :s["group_best"]].sum(2)
            best = torch.sort(good, dim=1, descending=True, stable=True).indices[:, :s["top_groups"]]
            allowed = torch.zeros((t, s["groups"]), dtype=torch.bool, device=x.device).scatter_(1, best, True)
            allowed = allowed[:, :, None].expand(-1, -1, e // s["groups"]).reshape(t, e)
            choice = torch.where(allowed, choice, torch.full_like(choice, -math.inf))
        ids = torch.sort(choice, dim=1, descending=True, stable=True).indices[:, :s["top"]]
        weights = torch.gather(_scores(x.float(), s["score"]), 1, ids)
        if s["renormalise"]:
            weights = weights / weights.sum(1, keepdim=True)
        weights = weights * s["scale"]
        if s["mask"] is not None:
            mask = s["mask"][i][:, None]
            ids, weights = torch.where(mask, ids, torch.full_like(ids, -1)), torch.where(mask, weights, torch.zeros_like(weights))
        ids_out.append(ids.to(s["ids"][i].dtype))
        weights_out.append(weights)
    return {"ids": ids_out, "weights": weights_out}


def _plain_route_grad(s):
    out = []
    for x, ids, up in zip(s["logits"], s["ids"], s["up"]):
        ids = ids.long()
        there = ids >= 0
        ids, up = ids.clamp(min=0), torch.where(there, up, torch.zeros_like(up)) * s["scale"]
        p = _scores(x.float(), s["score"])
        v = torch.gather(p, 1, ids) * there
        if s["renormalise"]:
            total = v.sum(1, keepdim=True)
            total = torch.where(total > 0, total, torch.ones_like(total))
            up = (up - (up * v).sum(1, keepdim=True) / total) / total * there
        d = torch.zeros_like(p).scatter_add_(1, ids, up)               # by the scores
        d = p * (d - (d * p).sum(1, keepdim=True)) if s["score"] == SOFTMAX else d * p * (1.0 - p)
        out.append(d.to(x.dtype))
    return out


def _plain_distill(s):
    loss_out, stats_out, t = [], [], s["temperature"]
    for i, (x, ids, teacher) in enumerate(zip(s["logits"], s["ids"], s["teacher"])):
        x = x.float()
        m = x.amax(1, keepdim=True)
        sum_t, sum_1 = torch.exp((x - m) / t).sum(1), torch.zeros_like(m[:, 0])
        y = teacher.float() / t
        y = y - y.amax(1, keepdim=True)
        log_q = y - torch.log(torch.exp(y).sum(1, keepdim=True))
        log_p = (torch.gather(x, 1, ids) - m) / t - torch.log(sum_t)[:, None]
        loss = t * t * (torch.exp(log_q) * (log_q - log_p)).sum(1)
        if s["labels"] is not None:
            label, sum_1 = s["labels"][i], torch.exp(x - m).sum(1)
            cross = torch.log(sum_1) - (torch.gather(x, 1, label.clamp(min=0)[:, None]) - m)[:, 0]
            loss = loss + s["label"] * torch.where(label >= 0, cross, torch.zeros_like(cross))
        stats = torch.stack([m[:, 0], sum_t, sum_1], 1)
        if s["mask"] is not None:
            loss = torch.where(s["mask"][i], loss, torch.zeros_like(loss))
            stats = torch.where(s["mask"][i][:, None], stats, torch.zeros_like(stats))
        loss_out.append(loss)
        stats_out.append(stats)
    return {"loss": loss_out, "stats": stats_out}


def _plain_distill_grad(s):
    out, t = [], s["temperature"]
    for i, (x, ids, teacher, stats) in enumerate(zip(s["logits"], s["ids"], s["teacher"], s["stats"])):
        m, sum_t, sum_1 = stats.unbind(1)
        x = x.float() - m[:, None]
        d = torch.exp(x / t) * (t / sum_t)[:, None]
        y = teacher.float() / t
        y = torch.exp(y - y.amax(1, keepdim=True))
        d.scatter_add_(1, ids, y * (-t / y.sum(1, keepdim=True)))
        if s["labels"] is not None:
            label = s["labels"][i]
            factor = s["label"] * (label >= 0).float()
            d += torch.exp(x) * (factor / sum_1)[:, None]
            d.scatter_add_(1, label.clamp(min=0)[:, None], -factor[:, None])
        d = d * s["up"]
        if s["mask"] is not None:
            d = torch.where(s["mask"][i][:, None], d, torch.zeros_like(d))
        out.append(d.to(s["logits"][i].dtype))
    return out


_PLAIN = {"route": _plain_route, "route_grad": _plain_route_grad, "distill": _plain_distill, "distill_grad": _plain_distill_grad}


# ---------------------------------------------------------------------------------------------- work and truth
def work(case):
    size, w = 4 if case["dtype"] == "f32" else 2, case["workers"]
    if case["kind"] in ("route", "route_grad"):
        t, e, k, id_size = case["tokens"], case["experts"], case["top"], 4 if case["ids"] == "i32" else 8
        valid = _counted_rows(t, case["masked"])
        if case["kind"] == "route":
            return {"bytes": w * (valid * e * size + t * k * (id_size + 4) + (t if case["masked"] else 0)) + (4 * e if case["biased"] else 0),
                    "flops": w * valid * e * (4 + 2 * k)}
        # the logits of the whole row only where the scores are its softmax, else those of the choices, or their weights
        read = valid * (e * size if case["score"] == SOFTMAX and not case["renormalise"] else k * (4 if case["score"] == SOFTMAX else size))
        return {"bytes": w * (read + t * e * size + t * k * id_size + valid * k * 4), "flops": w * valid * (10 * k + (8 * e if read > valid * k * 4 else 0))}
    r, v, k = case["rows"], case["vocab"], case["top"]
    valid, passes = _counted_rows(r, case["masked"]), 1 if case["label"] == 0.0 or case["temperature"] == 1.0 else 2
    small = valid * (k * (8 + size) + (8 if case["label"] else 0) + 12) + (r if case["masked"] else 0)
    if case["kind"] == "distill":
        return {"bytes": w * (valid * v * size + small + 4 * r), "flops": w * valid * v * (2 + 3 * passes)}
    return {"bytes": w * ((valid + r) * v * size + small) + 4, "flops": w * valid * v * (2 + 3 * passes)}


def exact(case, seed):
    """The definitions in 64 bits."""
    s = prepare(case, seed)
    return {"route": _exact_route, "route_grad": _exact_route_grad, "distill": _exact_distill, "distill_grad": _exact_distill_grad}[case["kind"]](s)


def _exact_route(s):
    ids_out, weights_out = [], []
    for w, x in enumerate(s["logits"]):
        z = x.double()
        p = torch.softmax(z, 1) if s["score"] == SOFTMAX else torch.sigmoid(z)
        left = z.clone() if s["bias"] is None and s["group_best"] == 1 else p + (0.0 if s["bias"] is None else s["bias"].double())
        tokens, experts = left.shape
        each = experts // s["groups"]
        if s["groups"] > 1:
            goodness = left.view(tokens, s["groups"], each).topk(s["group_best"], dim=2).values.sum(2)
            # a group stays if fewer than top_groups others are better, or as good and before it
            place = torch.arange(s["groups"], device=x.device)
            ahead = (goodness[:, None, :] > goodness[:, :, None]) | ((goodness[:, None, :] == goodness[:, :, None]) & (place[None, :] < place[:, None]))
            left[(ahead.sum(2) >= s["top_groups"]).repeat_interleave(each, 1)] = -math.inf
        ids = torch.empty((tokens, s["top"]), dtype=torch.int64, device=x.device)
        for j in range(s["top"]):
            ids[:, j] = (left == left.amax(1, keepdim=True)).to(torch.uint8).argmax(1)
            left.scatter_(1, ids[:, j:j + 1], -math.inf)
        weights = p.gather(1, ids)
        weights = s["scale"] * (weights / weights.sum(1, keepdim=True) if s["renormalise"] else weights)
        if s["mask"] is not None:
            ids[~s["mask"][w]] = -1
            weights[~s["mask"][w]] = 0.0
        ids_out.append(ids.to(s["ids"][w].dtype))
        weights_out.append(weights)
    return {"ids": ids_out, "weights": weights_out}


def _exact_route_grad(s):
    out = []
    for x, ids, up in zip(s["logits"], s["ids"], s["up"]):
        z, d = x.double(), torch.zeros(x.shape, dtype=torch.float64, device=x.device)
        rows = torch.nonzero(ids[:, 0] >= 0)[:, 0]
        z, ids, up = z[rows], ids[rows].long(), up[rows].double() * s["scale"]
        part = torch.zeros_like(z)
        if s["renormalise"]:
            chosen = z.gather(1, ids)
            logs = chosen if s["score"] == SOFTMAX else torch.nn.functional.logsigmoid(chosen)
            share = torch.softmax(logs, 1)
            by_log = share * (up - (share * up).sum(1, keepdim=True))
            part.scatter_add_(1, ids, by_log if s["score"] == SOFTMAX else by_log * torch.sigmoid(-chosen))
        elif s["score"] == SOFTMAX:
            p = torch.softmax(z, 1)
            part.scatter_add_(1, ids, up * p.gather(1, ids))
            part -= p * part.sum(1, keepdim=True)
        else:
            chosen = z.gather(1, ids)
            part.scatter_add_(1, ids, up * torch.sigmoid(chosen) * torch.sigmoid(-chosen))
        d[rows] = part
        out.append(d)
    return out


def _pieces(s):
    """The rows of every worker, so many at a time that 64 bits fit."""
    for w, x in enumerate(s["logits"]):
        step = max(1, (1 << 26) // x.shape[1])
        for a in range(0, x.shape[0], step):
            yield w, slice(a, min(x.shape[0], a + step))


def _exact_distill(s):
    t, loss, stats = s["temperature"], [[] for _ in s["logits"]], [[] for _ in s["logits"]]
    for w, at in _pieces(s):
        x = s["logits"][w][at].double()
        m = x.amax(1)
        log_q = torch.log_softmax(s["teacher"][w][at].double() / t, 1)
        lse = torch.logsumexp(x / t, 1)
        value = t * t * (log_q.exp() * (log_q + lse[:, None] - x.gather(1, s["ids"][w][at]) / t)).sum(1)
        sum_1 = torch.zeros_like(m)
        if s["labels"] is not None:
            label, lse_1 = s["labels"][w][at], torch.logsumexp(x, 1)
            sum_1 = (lse_1 - m).exp()
            value = value + s["label"] * (lse_1 - x.gather(1, label.clamp(min=0)[:, None])[:, 0]) * (label >= 0)
        of_row = torch.stack([m, (lse - m / t).exp(), sum_1], 1)
        if s["mask"] is not None:
            value, of_row = value * s["mask"][w][at], of_row * s["mask"][w][at][:, None]
        loss[w].append(value)
        stats[w].append(of_row)
    return {"loss": [torch.cat(c) for c in loss], "stats": [torch.cat(c) for c in stats]}


def _exact_distill_grad(s):
    t, up, out = s["temperature"], float(s["up"]), [torch.empty(x.shape, dtype=torch.float64, device=x.device) for x in s["logits"]]
    for w, at in _pieces(s):
        x, (m, sum_t, sum_1) = s["logits"][w][at].double(), s["stats"][w][at].double().unbind(1)
        d = t * torch.exp((x - m[:, None]) / t - torch.log(sum_t)[:, None])
        d.scatter_add_(1, s["ids"][w][at], -t * torch.softmax(s["teacher"][w][at].double() / t, 1))
        if s["labels"] is not None:
            label = s["labels"][w][at]
            rows = torch.nonzero(label >= 0)[:, 0]
            part = torch.exp(x[rows] - m[rows, None]) / sum_1[rows, None]
            part.scatter_add_(1, label[rows, None], torch.full((rows.numel(), 1), -1.0, dtype=torch.float64, device=x.device))
            d[rows] += s["label"] * part
        if s["mask"] is not None:
            d[~s["mask"][w][at]] = 0.0
        out[w][at] = d * up
    return out
