"""The operators around a communication round whose speed is looked after: what a training loop runs on the averaged gradients
(global norm and clipping factor, AdamW over many tensors) and the balance loss of a mixture of experts, whose statistics are
sums over all workers' tokens.

A case is one call of one operator ("kind"):

  norm      global gradient norm over a list of tensors, and the factor that clips it.
  adamw     one AdamW step over a list of tensors.  states = 32: both moments in fp32; 8: in blocks of 256 elements as E4M3
            codes with one fp32 scale, the first moment rounded to nearest, the root of the second one stochastically.
            form "f32": fp32 parameters and gradients; "mixed": fp32 parameters, bf16 gradients, and a bf16 copy of the
            parameters is written; "bf16": bf16 parameters (stochastically rounded) and gradients.
  balance   forward of the balance loss of `workers` workers' tokens: per-expert counts and probability sums, the loss and
            its derivative with respect to the probability sums.
  balance_grad   its backward: gradient of the router's logits.

Where `own` is false the operators are computed in plain torch operations in 32 bits.  AdamW is defined bit for bit (one
rounding per operation in a fixed order; the random numbers are a hash of the seed and the element's place), the others by
their formula.
"""
import math
import random

import torch

own = False

BLOCK = 256                  # elements of one scale, and the quantum of a tensor's place in its storage
LARGEST = 9.4e9              # bytes: no drawn case needs more than the largest listed one
BETA1, BETA2, EPS, LR, DECAY = 0.9, 0.95, 1e-8, 1e-3, 0.1
BETA2_32 = 0.999
MAX_NORM = 1.0
ALPHA = 0.01                 # weight of the balance loss


def listed():
    return [
        # one small module's gradients: the call itself counts
        dict(name="norm_small", kind="norm", n=40961, dtype="f32"),
        # BERT-large-sized gradients, once per step before the optimizer
        dict(name="norm_bert_large", kind="norm", n=335141888, dtype="f32"),
        # an adapter's or a small module's step: latency
        dict(name="adamw32_small", kind="adamw", n=40961, form="f32", states=32),
        # ResNet-50-sized model in full precision
        dict(name="adamw32_resnet50", kind="adamw", n=25557032, form="f32", states=32),
        # BERT-large-sized model in mixed precision: fp32 parameters, bf16 gradients, bf16 copy for the next forward; the largest
        dict(name="adamw32_bert_large_mixed", kind="adamw", n=335141888, form="mixed", states=32),
        # the small module with states in 8 bits
        dict(name="adamw8_small", kind="adamw", n=40961, form="f32", states=8),
        # BERT-base-sized model, mixed precision, states in 8 bits
        dict(name="adamw8_bert_base_mixed", kind="adamw", n=109482241, form="mixed", states=8),
        # the least memory a step can do with: bf16 parameters without an fp32 copy, states in 8 bits
        dict(name="adamw8_bert_large_bf16", kind="adamw", n=335141888, form="bf16", states=8),
        # one micro-batch of a small mixture
        dict(name="balance_small", kind="balance", workers=1, tokens=500, experts=8, top=2, dtype="f32", masked=False),
        # eight workers' batches through 64 experts, padded sequences; the balance is that of the whole batch
        dict(name="balance_8_workers", kind="balance", workers=8, tokens=32768, experts=64, top=6, dtype="bf16", masked=True),
        # four workers with an odd number of experts in full precision
        dict(name="balance_grad_odd", kind="balance_grad", workers=4, tokens=4099, experts=60, top=4, dtype="f32", masked=True),
        # a long batch through many experts
        dict(name="balance_grad_large", kind="balance_grad", workers=1, tokens=524288, experts=256, top=8, dtype="bf16", masked=False),
    ]


def draw(rng):
    """One more case of the same ranges: any kind, sizes spread over their logarithm, odd ones among them."""
    while True:
        kind = rng.choice(["norm", "adamw", "adamw", "balance", "balance_grad"])
        if kind in ("norm", "adamw"):
            n = int(2.0 ** rng.uniform(8.0, 28.3))
            case = dict(kind=kind, n=rng.choice([n, n | 1, n // 256 * 256]))
            if kind == "norm":
                case.update(dtype=rng.choice(["f32", "bf16"]))
            else:
                case.update(form=rng.choice(["f32", "mixed", "bf16"]), states=rng.choice([8, 32]))
        else:
            experts = rng.choice([2, 4, 7, 8, 16, 32, 60, 64, 72, 100, 128, 160, 256, 384, 512])
            case = dict(kind=kind, workers=rng.choice([1, 1, 2, 3, 4, 8]), tokens=int(2.0 ** rng.uniform(0.0, 19.0)), experts=experts,
                        top=min(experts, rng.choice([1, 2, 2, 4, 6, 8])), dtype=rng.choice(["f32", "bf16", "bf16", "f16"]),
                        masked=rng.random() < 0.5)
            if case["tokens"] * case["workers"] * experts > 1 << 27:
                continue
        if work(case)["bytes"] <= LARGEST:
            return case


# ---------------------------------------------------------------------------------------------- inputs
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
F8 = torch.float8_e4m3fn


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(n, g, sigma=1.0):
    return torch.empty(n, dtype=torch.float32, device="cuda").normal_(0.0, sigma, generator=g)


def _sizes(n):
    """Sizes of a model's tensors that sum to n: matrices of very different sizes, each with two short vectors."""
    rng, sizes, left = random.Random(n), [], n
    largest = max(9.0, min(22.5, math.log2(n) - 3.0))
    while left > 0:
        for s in (int(2.0 ** rng.uniform(7.0, largest)), rng.choice([64, 256, 768, 1024, 2048]), rng.choice([1, 65, 255, 1000, 1024])):
            if left > 0:
                sizes.append(min(s, left))
                left -= sizes[-1]
    return sizes


class _Places:
    """Where a model's tensors lie: each at a place of its own in one storage per kind of data (zeros between them), as an
    allocator gives them.  The storages are what is compared; the operators get the tensors."""

    def __init__(self, n):
        self.sizes = _sizes(n)
        self.starts, at = [], 0
        for s in self.sizes:
            self.starts.append(at)
            at += (s + BLOCK - 1) // BLOCK * BLOCK
        self.total = at
        tensor, place = [], []
        for t, s in enumerate(self.sizes):
            blocks = (s + BLOCK - 1) // BLOCK
            tensor.append(torch.full((blocks,), t, dtype=torch.int64))
            place.append(torch.arange(blocks, dtype=torch.int64))
        self.tensor, self.place = torch.cat(tensor).cuda(), torch.cat(place).cuda()     # of every block: its tensor, its index there
        self.last = torch.tensor(self.sizes, dtype=torch.int64).cuda()

    def here(self):
        """Of every element of a storage: whether it belongs to a tensor."""
        left = self.last[self.tensor] - self.place * BLOCK
        return (torch.arange(BLOCK, device="cuda")[None, :] < left[:, None]).view(-1)

    def parts(self, storage, per=1):
        """The tensors of a storage that holds one value for `per` elements."""
        return [storage[a // per:a // per + (s + per - 1) // per] for a, s in zip(self.starts, self.sizes)]


def _decays(count):
    """Vectors (biases, norms) are not decayed."""
    return [1.0 if t % 3 == 0 else 0.0 for t in range(count)]


def prepare(case, seed):
    g = _gen(seed)
    return {"norm": _prepare_norm, "adamw": _prepare_adamw, "balance": _prepare_balance, "balance_grad": _prepare_balance}[case["kind"]](case, g, seed)


def _grads(places, dtype, g):
    """Gradients whose size differs from tensor to tensor."""
    scale = (10.0 ** torch.empty(len(places.sizes), device="cuda").uniform_(-4.0, -2.0, generator=g))[places.tensor]
    x = _normal(places.total, g).view(-1, BLOCK).mul_(scale[:, None]).view(-1)
    return x.mul_(places.here()).to(TYPES[dtype])


def _plan(s, places, **more):
    import paper_2107_01499_amd as bg
    ws = torch.empty(bg.bagua_tensor_plan_bytes(places.sizes), dtype=torch.uint8, device="cuda")
    s["plan"] = bg.bagua_tensor_plan(places.parts(s["g"]), ws, **more)


def _prepare_norm(case, g, seed):
    places = _Places(case["n"])
    s = dict(kind="norm", places=places, g=_grads(places, case["dtype"], g), out=torch.zeros(2, device="cuda"))
    if own:
        _plan(s, places)
    return s


def _prepare_adamw(case, g, seed):
    places = _Places(case["n"])
    form, bits = case["form"], case["states"]
    here = places.here()
    s = dict(kind="adamw", form=form, bits=bits, places=places, step=1000 + seed % 1000, beta2=BETA2_32 if bits == 32 else BETA2,
             g=_grads(places, "f32" if form == "f32" else "bf16", g), p=_normal(places.total, g, 0.02).mul_(here))
    if form == "bf16":
        s["p"] = s["p"].to(torch.bfloat16)
    if form == "mixed":
        s["copy"] = s["p"].to(torch.bfloat16)
    # moments as they are in the middle of a run: of the size of the gradients
    if bits == 32:
        size = s["g"].float().square_().view(-1, BLOCK).mean(1, keepdim=True)
        s["m"] = _normal(places.total, g, 0.3).view(-1, BLOCK).mul_(size.sqrt()).view(-1).mul_(here)
        s["v"] = _normal(places.total, g).square_().add_(0.05).view(-1, BLOCK).mul_(size).view(-1).mul_(here)
    else:
        blocks = places.total // BLOCK
        size = s["g"].float().square_().view(-1, BLOCK).mean(1).sqrt_()
        s["m"] = _normal(places.total, g, 100.0).clamp_(-448.0, 448.0).mul_(here).to(F8)
        s["v"] = _normal(places.total, g, 100.0).abs_().clamp_(1.0, 448.0).mul_(here).to(F8)
        s["ms"] = torch.empty(blocks, device="cuda").uniform_(0.5, 1.5, generator=g).mul_(size * 0.003)
        s["vs"] = torch.empty(blocks, device="cuda").uniform_(0.5, 1.5, generator=g).mul_(size * 0.010)
    s["clip"] = torch.tensor([1.37, 0.7299265], device="cuda")      # what the norm's call has left: the norm and the factor
    decays = _decays(len(places.sizes))
    s["decay"] = torch.tensor(decays, device="cuda")
    if own:
        more = dict(params=places.parts(s["p"]), m=places.parts(s["m"]), v=places.parts(s["v"]), decay=decays)
        if form == "mixed":
            more.update(copies=places.parts(s["copy"]))
        if bits == 8:
            more.update(m_scales=places.parts(s["ms"], BLOCK), v_scales=places.parts(s["vs"], BLOCK))
        _plan(s, places, **more)
    return s


def _valid(case):
    """How many of a worker's tokens are no padding."""
    t = case["tokens"]
    return t - t // 8 if case["masked"] else t


def _prepare_balance(case, g, seed):
    w, t, e, k = case["workers"], case["tokens"], case["experts"], case["top"]
    s = dict(kind=case["kind"], experts=e, top=k, logits=[], ids=[], mask=[] if case["masked"] else None)
    liking = _normal(e, g, 0.7)                        # some experts are more popular than others
    for _ in range(w):
        x = (_normal(t * e, g).view(t, e) * 1.5 + liking).to(TYPES[case["dtype"]])
        ids = torch.topk(x.float() + 0.1 * _normal(t * e, g).view(t, e), k, dim=1).indices
        ids[torch.rand(t, k, device="cuda", generator=g) < 0.02] = -1        # choices beyond an expert's capacity were dropped
        s["logits"].append(x)
        s["ids"].append(ids)
        if case["masked"]:                             # padding at the ends of sequences
            order = torch.rand(max(1, t // 64 + 1), device="cuda", generator=g).repeat_interleave(64)[:t].argsort(stable=True)
            mask = torch.zeros(t, dtype=torch.bool, device="cuda")
            mask[order[:_valid(case)]] = True
            s["mask"].append(mask)
    if s["kind"] == "balance":
        s.update(counts=torch.zeros(e + 1, dtype=torch.int32, device="cuda"), prob=torch.zeros(e, device="cuda"),
                 loss=torch.zeros(1, device="cuda"), weight=torch.zeros(e, device="cuda"))
        if own:
            import paper_2107_01499_amd as bg
            s["ws"] = torch.zeros(bg.bagua_balance_workspace_bytes(e), dtype=torch.uint8, device="cuda")
    else:
        # what the forward has left, and the gradient that arrives at the loss
        total = float(w * _valid(case))
        load = torch.rand(e, device="cuda", generator=g) + 0.2
        s.update(weight=load / load.sum() * (ALPHA * e / max(total, 1.0)), up=torch.full((1,), 1024.0, device="cuda"),
                 out=[torch.zeros_like(x) for x in s["logits"]])
    return s


# ---------------------------------------------------------------------------------------------- one call
def run(state):
    if own:
        return _OWN[state["kind"]](state)
    return _PLAIN[state["kind"]](state)


def _updated(s):
    return {k: s[k] for k in ("p", "m", "v", "ms", "vs", "copy") if k in s}


def _own_norm(s):
    import paper_2107_01499_amd as bg
    bg.bagua_grad_norm(s["plan"], s["out"], MAX_NORM)
    return s["out"]


def _own_adamw(s):
    import paper_2107_01499_amd as bg
    s["step"] += 1
    bg.bagua_adamw_step(s["plan"], s["step"], LR, BETA1, s["beta2"], EPS, DECAY, clip=s["clip"], seed=s["step"])
    return _updated(s)


def _own_balance(s):
    import paper_2107_01499_amd as bg
    bg.bagua_balance_stats(s["logits"], s["ids"], s["mask"], s["counts"], s["prob"], s["ws"], ALPHA, s["loss"], s["weight"])
    return {k: s[k] for k in ("counts", "prob", "loss", "weight")}


def _own_balance_grad(s):
    import paper_2107_01499_amd as bg
    bg.bagua_balance_grad(s["logits"], s["mask"], s["weight"], s["up"], s["out"])
    return s["out"]


_OWN = {"norm": _own_norm, "adamw": _own_adamw, "balance": _own_balance, "balance_grad": _own_balance_grad}


# ---------------------------------------------------------------------------------------------- plain forms
def _plain_norm(s):
    norm = s["g"].float().square().sum().sqrt()
    return torch.stack([norm, torch.clamp(MAX_NORM / (norm + 1e-6), max=1.0)])


GOLDEN, ROOT2, ROOT3, LOW = 0x9E3779B9, 0x6A09E667, 0xBB67AE85, 0xFFFFFFFF     # fractions of the golden ratio and two roots, 32 bits


def _mix(x):
    """A hash of 32-bit numbers (held in 64 bits)."""
    x = ((x ^ (x >> 16)) * ROOT2) & LOW
    x = ((x ^ (x >> 15)) * ROOT3) & LOW
    return x ^ (x >> 16)


def _hash(places, seed):
    """One 32-bit random number for every four consecutive elements of a tensor."""
    base = _mix((places.tensor * GOLDEN + seed) & LOW)
    four = places.place[:, None] * (BLOCK // 4) + torch.arange(BLOCK // 4, device="cuda")
    return _mix((four * GOLDEN + base[:, None]) & LOW)


def _random_bits(h, bits):
    """`bits` random bits for each element: the number of its four, turned by eight for each place."""
    at = torch.arange(4, device=h.device) * 8
    turned = ((h[..., None] << at) | (h[..., None] >> (32 - at))) & LOW
    return (turned >> (32 - bits)).view(h.shape[0], -1)


def _quantise(x, scale_of):
    """Scale and reciprocal of blocks whose largest magnitude is scale_of; a block that is zero (or nearly) gets 0."""
    scale = scale_of * (1.0 / 448.0)
    scale = torch.where(scale >= 2.0 ** -126, scale, torch.zeros_like(scale))
    inverse = torch.where(scale > 0, torch.ones_like(scale) / scale, torch.zeros_like(scale))
    return scale, x * inverse[:, None]


def _plain_adamw(s):
    s["step"] += 1
    step, places = s["step"], s["places"]
    b1, b2 = BETA1, s["beta2"]
    g = s["g"].float() * s["clip"][1]
    p = s["p"].float()
    if s["bits"] == 8:
        m = (s["m"].float().view(-1, BLOCK) * s["ms"][:, None]).view(-1)
        r = (s["v"].float().view(-1, BLOCK) * s["vs"][:, None]).view(-1)
        v = r * r
    else:
        m, v = s["m"], s["v"]
    m = m * b1 + g * (1.0 - b1)
    v = v * b2 + (g * g) * (1.0 - b2)
    r = v.sqrt()
    denominator = r * (1.0 / math.sqrt(1.0 - b2 ** step)) + EPS
    update = (m / denominator) * (LR / (1.0 - b1 ** step))
    decay = (s["decay"] * (LR * DECAY))[places.tensor]
    p = p - (update.view(-1, BLOCK) + p.view(-1, BLOCK) * decay[:, None]).view(-1)
    if s["bits"] == 8 or s["form"] == "bf16":
        h = _hash(places, step)
    if s["bits"] == 8:
        m, r = m.view(-1, BLOCK), r.view(-1, BLOCK)
        scale, code = _quantise(m, m.abs().amax(1))
        s["ms"].copy_(scale)
        s["m"].copy_(code.to(F8).view(-1))
        scale, code = _quantise(r, r.amax(1))
        s["vs"].copy_(scale)
        bits = (code * 2.0 ** -120).view(torch.int32) + _random_bits(h, 20).to(torch.int32)
        code = torch.where(r > 0, (bits >> 20).clamp(1, 126), torch.zeros_like(bits))      # a second moment above zero stays above it
        s["v"].copy_(code.to(torch.uint8).view(F8).view(-1))
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    if s["form"] == "bf16":
        bits = (p.view(torch.int32).to(torch.int64) & LOW) + _random_bits(_mix((h + GOLDEN) & LOW), 16).view(-1)
        s["p"].copy_(torch.where(places.here(), bits >> 16, torch.zeros_like(bits)).to(torch.int16).view(torch.bfloat16))
    else:
        s["p"].copy_(p)
    if s["form"] == "mixed":
        s["copy"].copy_(p)
    return _updated(s)


def _probabilities(x, mask):
    x = x.float()
    x = torch.exp(x - x.amax(1, keepdim=True))
    x = x / x.sum(1, keepdim=True)
    return x if mask is None else torch.where(mask[:, None], x, torch.zeros_like(x))


def _counted(ids, mask, experts):
    """How often each expert was chosen; many rows of counters, for they are added to one at a time."""
    ids = ids if mask is None else torch.where(mask[:, None], ids, torch.full_like(ids, -1))
    rows = 1024
    at = torch.arange(ids.shape[0], device=ids.device)[:, None] % rows * (experts + 1) + torch.where(ids < 0, torch.full_like(ids, experts), ids)
    counts = torch.zeros(rows * (experts + 1), dtype=torch.int32, device=ids.device)
    counts.scatter_add_(0, at.view(-1), torch.ones(1, dtype=torch.int32, device=ids.device).expand(at.numel()))
    counts = counts.view(rows, experts + 1).sum(0, dtype=torch.int32)
    counts[experts] = ids.shape[0] if mask is None else mask.sum()
    return counts


def _masks(s):
    return s["mask"] or [None] * len(s["logits"])


def _plain_balance(s):
    e, k = s["experts"], s["top"]
    prob = torch.stack([_probabilities(x, m).sum(0) for x, m in zip(s["logits"], _masks(s))]).sum(0)
    counts = torch.stack([_counted(i, m, e) for i, m in zip(s["ids"], _masks(s))]).sum(0, dtype=torch.int32)
    tokens = counts[e].float().clamp(min=1.0)
    weight = counts[:e].float() * (ALPHA * e / k) / tokens / tokens
    return {"counts": counts, "prob": prob, "loss": (weight * prob).sum().view(1), "weight": weight}


def _plain_balance_grad(s):
    def one(x, mask):
        p = _probabilities(x, mask)
        return (p * (s["weight"] - (p * s["weight"]).sum(1, keepdim=True)) * s["up"]).to(x.dtype)
    return [one(x, m) for x, m in zip(s["logits"], _masks(s))]


_PLAIN = {"norm": _plain_norm, "adamw": _plain_adamw, "balance": _plain_balance, "balance_grad": _plain_balance_grad}


# ---------------------------------------------------------------------------------------------- work and truth
def work(case):
    if case["kind"] == "norm":
        return {"bytes": case["n"] * (4 if case["dtype"] == "f32" else 2) + 8, "flops": 2 * case["n"]}
    if case["kind"] == "adamw":
        per = {"f32": 8 + 4, "mixed": 8 + 2 + 2, "bf16": 4 + 2}[case["form"]] + (16 if case["states"] == 32 else 4 + 16 / BLOCK)
        return {"bytes": case["n"] * per, "flops": 17 * case["n"]}
    w, t, e, k = case["workers"], case["tokens"], case["experts"], case["top"]
    size, valid = 4 if case["dtype"] == "f32" else 2, _valid(case)
    seen = t if case["masked"] else 0
    if case["kind"] == "balance":
        return {"bytes": w * (valid * (e * size + k * 8) + seen) + 12 * e + 8, "flops": 6 * w * valid * e}
    return {"bytes": w * ((valid + t) * e * size + seen) + 4 * e + 4, "flops": 9 * w * valid * e}


def exact(case, seed):
    """The definitions in 64 bits."""
    s = prepare(case, seed)
    return {"norm": _exact_norm, "adamw": _exact_adamw, "balance": _exact_balance, "balance_grad": _exact_balance_grad}[case["kind"]](s)


def _exact_norm(s):
    norm = math.sqrt(sum(float(torch.dot(x, x)) for x in (c.double() for c in s["g"].split(1 << 26))))
    return torch.tensor([norm, min(1.0, MAX_NORM / (norm + 1e-6))], dtype=torch.float64)


def _code_values():
    """The 127 magnitudes that E4M3 has, by code: 2^(e-7) (1 + f/8), below 2^-6 steps of 2^-9."""
    return torch.tensor([c * 2.0 ** -9 if c < 8 else (8 + c % 8) * 2.0 ** (c // 8 - 10) for c in range(127)], dtype=torch.float64, device="cuda")


def _exact_adamw(s):
    t, b1, b2, values = s["step"] + 1, BETA1, s["beta2"], _code_values()
    out = {k: [] for k in _updated(s)}
    factor = float(s["clip"][1])
    for first in range(0, s["places"].total // BLOCK, 1 << 17):
        blocks = slice(first, first + (1 << 17))
        part = lambda k: s[k].view(-1, BLOCK)[blocks].double()  # noqa: E731
        g, p = part("g") * factor, part("p")
        m, v = part("m"), part("v")
        if s["bits"] == 8:
            m, v = m * s["ms"][blocks, None].double(), (v * s["vs"][blocks, None].double()) ** 2
        m = b1 * m + (1 - b1) * g
        v = b2 * v + (1 - b2) * g * g
        wd = DECAY * s["decay"].double()[s["places"].tensor[blocks]]
        p = p - LR * ((m / (1 - b1 ** t)) / ((v / (1 - b2 ** t)).sqrt() + EPS) + wd[:, None] * p)
        if s["bits"] == 8 or s["form"] == "bf16":
            spots = _Spots(s["places"].tensor[blocks], s["places"].place[blocks])
            h = _hash(spots, t)
        if s["bits"] == 8:
            r = v.sqrt()
            ms, vs = m.abs().amax(1) / 448, r.amax(1) / 448
            out["ms"].append(ms)
            out["vs"].append(vs)
            y = (m.abs() / ms.clamp(min=1e-300)[:, None]).clamp(max=448.0)
            hi = torch.searchsorted(values, y).clamp(max=126)
            lo = (hi - 1).clamp(min=0)
            near = torch.where(y - values[lo] < values[hi] - y, lo, hi)
            near = torch.where((y - values[lo] == values[hi] - y) & (lo % 2 == 0), lo, near)
            out["m"].append(values[near] * m.sign())
            y = (r / vs.clamp(min=1e-300)[:, None]).clamp(max=448.0)
            lo = (torch.searchsorted(values, y, right=True) - 1).clamp(0, 125)
            up = (y - values[lo]) / (values[lo + 1] - values[lo]) + _random_bits(h, 20).double() / 2 ** 20 >= 1
            out["v"].append(torch.where(r > 0, values[torch.where(up, lo + 1, lo).clamp(min=1)], torch.zeros_like(r)))
        else:
            out["m"].append(m)
            out["v"].append(v)
        if s["form"] == "bf16":        # the value between two bf16 numbers goes up where the random bits reach over what it lacks
            size = p.abs().clamp(min=2.0 ** -126).log2().floor().exp2() * 2.0 ** -7
            q = p.abs() / size
            q = (q.floor() + ((q - q.floor()) + _random_bits(_mix((h + GOLDEN) & LOW), 16).double() / 2 ** 16 >= 1)) * size * p.sign()
            out["p"].append(torch.where(p == 0, p, q))
        else:
            out["p"].append(p)
        if s["form"] == "mixed":
            out["copy"].append(p.to(torch.float32).to(torch.bfloat16).double())
    return {k: torch.cat([x.reshape(-1) for x in v]) for k, v in out.items()}


class _Spots:
    def __init__(self, tensor, place):
        self.tensor, self.place = tensor, place


def _exact_balance(s):
    e, k = s["experts"], s["top"]
    prob, counts, tokens = torch.zeros(e, dtype=torch.float64, device="cuda"), torch.zeros(e, dtype=torch.int64, device="cuda"), 0
    for x, ids, mask in zip(s["logits"], s["ids"], _masks(s)):
        x, ids = (x, ids) if mask is None else (x[mask], ids[mask])
        prob += torch.softmax(x.double(), 1).sum(0)
        counts += torch.bincount(ids[ids >= 0], minlength=e)
        tokens += x.shape[0]
    weight = ALPHA * e * counts.double() / (k * tokens) / tokens if tokens else torch.zeros_like(prob)
    return {"counts": torch.cat([counts, torch.tensor([tokens], device="cuda")]).to(torch.int32), "prob": prob, "loss": (weight * prob).sum().view(1),
            "weight": weight}


def _exact_balance_grad(s):
    out = []
    for x, mask in zip(s["logits"], _masks(s)):
        p = torch.softmax(x.double(), 1)
        d = p * (s["weight"].double() - (p @ s["weight"].double())[:, None]) * float(s["up"])
        out.append(d if mask is None else torch.where(mask[:, None], d, torch.zeros_like(d)))
    return out
