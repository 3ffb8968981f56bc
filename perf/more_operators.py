"""Workloads of the expert layer's operators and of dropout: what a rank computes between
the token table and the gradients that the modelled collectives carry.

Every case is one call of a public entry point on tensors that are already in HBM.
Five kinds, forward or, where `grad` is set, backward:

  gate     themis_expert_gate: the k largest of a token's logits and their softmax;
           themis_expert_gate_grad
  sort     themis_expert_sort: tokens in the order of their experts, packed or in
           fixed buffers of `capacity` rows for every expert
  there    themis_expert_dispatch: rows in that order; its gradient is
           themis_expert_combine without weights
  back     themis_expert_combine: the weighted sum of a token's rows;
           themis_expert_combine_grad
  dropout  themis_dropout: with what it is added to, or, backward, alone

Fields of a case:
  tokens, width, experts, k   tokens, elements of a row, experts, experts of a token
  type, to    element types of what is read and of what is written
  index       gate, sort: type of the expert numbers
  over        gate: the softmax is over the "chosen" logits or over "all"
  masked      gate: share of the logits that are -inf (experts out of a token's reach)
  capacity    rows of an expert's buffer over the mean load; 0: packed
  weights     back: type of the weights
  add         back: added to what the output holds (a residual, a shared expert);
              dropout: added to another tensor
  p           dropout: probability
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16,
         "i32": torch.int32, "i64": torch.int64}
SIZE = {"f32": 4, "bf16": 2, "f16": 2, "i32": 4, "i64": 8}


def listed():
    return [
        # the smallest call: one token of a decoding step
        dict(name="gate of one token", kind="gate", grad=False, tokens=1, experts=64, k=2,
             type="bf16", to="f32", index="i32", over="chosen", masked=0.0),
        # a training step on many experts, half of which a token may not choose
        dict(name="gate of a large step", kind="gate", grad=False, tokens=65536, experts=256, k=8,
             type="bf16", to="f32", index="i32", over="chosen", masked=0.5),
        # odd sizes; probabilities over all experts, so every logit has a gradient
        dict(name="gate, odd, gradient", kind="gate", grad=True, tokens=8191, experts=60, k=4,
             type="f32", to="f32", index="i64", over="all", masked=0.0),
        # a sequence into fixed buffers of an expert-parallel exchange
        dict(name="sort of a sequence", kind="sort", grad=False, tokens=4096, experts=8, k=2,
             index="i64", capacity=1.25),
        # the largest step's tokens, packed
        dict(name="sort of a large step", kind="sort", grad=False, tokens=131072, experts=256, k=8,
             index="i32", capacity=0),
        # rows of a large step, eight copies each: the most that is written
        dict(name="there, large", kind="there", grad=False, tokens=16384, width=4096, experts=128,
             k=8, type="bf16", to="bf16", capacity=0),
        # odd sizes, gradients of half precision into binary32, some tokens dropped
        dict(name="there, odd, gradient", kind="there", grad=True, tokens=10007, width=1001,
             experts=13, k=3, type="f16", to="f32", capacity=1.0),
        # one token of a decoding step
        dict(name="back, one token", kind="back", grad=False, tokens=1, width=4096, experts=64, k=8,
             type="bf16", to="bf16", weights="f32", capacity=0, add=False),
        # a training step, added to the residual
        dict(name="back, large", kind="back", grad=False, tokens=32768, width=2048, experts=64, k=8,
             type="bf16", to="bf16", weights="f32", capacity=0, add=True),
        # gradients of the experts' rows and of the weights, fixed buffers
        dict(name="back, gradient", kind="back", grad=True, tokens=16384, width=4096, experts=8, k=2,
             type="bf16", to="bf16", weights="f32", capacity=1.25),
        # odd rows of an ordinary batch on their way into the residual
        dict(name="dropout, odd", kind="dropout", grad=False, tokens=4099, width=1001, type="f32",
             to="f32", p=0.1, add=True),
        # the gradient of a large step's activations
        dict(name="dropout, gradient", kind="dropout", grad=True, tokens=65536, width=4096,
             type="bf16", to="bf16", p=0.1, add=False),
    ]


def _log_int(rng, lo, hi):
    """An integer of [lo, hi], uniform over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _size(rng, lo, hi):
    """A size of [lo, hi]: a power of two, odd, or eight times an odd number."""
    n = _log_int(rng, lo, hi)
    kind = rng.choice(("power", "odd", "eight"))
    if kind == "power":
        n = 1 << int(math.log2(n) + 0.5)
        return n if lo <= n <= hi else lo
    if kind == "eight" and n >= 8 * max(lo, 1):
        return 8 * (n // 8 | 1) if 8 * (n // 8 | 1) <= hi else 8 * (n // 8 - 1 | 1)
    return n | 1 if n | 1 <= hi else max(lo, (n - 2) | 1)


def draw(rng):
    kind = rng.choices(("gate", "sort", "there", "back", "dropout"), (24, 16, 20, 24, 16))[0]
    case = dict(kind=kind, grad=kind != "sort" and rng.random() < 0.5)
    kinds = rng.choice((("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("f32", "bf16"),
                        ("bf16", "f32"), ("f16", "f32")))
    if kind != "sort":
        case.update(type=kinds[0], to=kinds[1])
    if kind == "dropout":
        width = _size(rng, 32, 8192)
        case.update(width=width, tokens=_size(rng, 1, min(131072, (1 << 27) // width)),
                    p=rng.choice((0.05, 0.1, 0.3, 0.5)), add=not case["grad"] and rng.random() < 0.5)
        return case
    experts = _size(rng, 2, 512)
    k = min(experts, rng.choice((1, 2, 2, 3, 4, 6, 8, 8)))
    case.update(experts=experts, k=k)
    if kind == "gate":
        case.update(tokens=_size(rng, 1, min(131072, (1 << 24) // experts)),
                    index=rng.choice(("i32", "i64")), over=rng.choice(("chosen", "all")),
                    masked=rng.choice((0.0, 0.0, 0.25, 0.5)))
        return case
    case["capacity"] = rng.choice((0, 0, 1.0, 1.25, 2.0))
    if kind == "sort":
        case.update(tokens=_size(rng, 1, 131072), index=rng.choice(("i32", "i64")))
        return case
    width = _size(rng, 32, 8192)
    case.update(width=width, tokens=_size(rng, 1, min(131072, (1 << 27) // (k * width))))
    if kind == "back":
        case["weights"] = rng.choice(("f32", "f32", "bf16"))
        if not case["grad"]:
            case["add"] = rng.random() < 0.4
    return case


def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _capacity(case):
    """Rows of an expert's buffer; 0: none, the rows are packed."""
    return math.ceil(case["capacity"] * case["tokens"] * case["k"] / case["experts"])


def _slots(case):
    return case["experts"] * _capacity(case) if case["capacity"] else case["tokens"] * case["k"]


def _logits(case, gen):
    """Gate logits: experts differ in how often they are chosen."""
    bias = torch.randn(case["experts"], generator=gen, device=DEV).mul_(0.7)
    return torch.randn((case["tokens"], case["experts"]), generator=gen, device=DEV).mul_(1.5).add_(bias)


def _top(logits, k):
    """The k largest of every row, largest first, the lowest index among equal ones; -1 for -inf."""
    live = logits.clone()
    number = torch.arange(logits.shape[1], device=DEV)
    values, experts = [], []
    for _ in range(k):
        top = live.amax(-1, keepdim=True)
        at = torch.where(live == top, number, logits.shape[1]).amin(-1, keepdim=True)
        live.scatter_(1, at, -math.inf)
        values.append(top)
        experts.append(torch.where(top == -math.inf, -1, at))
    return torch.cat(values, 1), torch.cat(experts, 1)


def _order(experts, n_experts, capacity, slots):
    """place[token][j]: the slot of a token's j-th expert, -1 for none; counts of the experts;
    the first slot of each, and the end; source[slot]: token * k + j, -1 for none."""
    flat = experts.reshape(-1).long()
    key, sorted_ = torch.sort(torch.where((flat < 0) | (flat >= n_experts), n_experts, flat), stable=True)
    number = torch.arange(n_experts + 1, device=DEV)
    first = torch.searchsorted(key, number)
    counts = first[1:] - first[:-1]
    rank = torch.arange(key.numel(), device=DEV) - first[key]
    if capacity:
        starts, slot = number * capacity, key * capacity + rank
        slot = torch.where((key < n_experts) & (rank < capacity), slot, -1)
    else:
        starts, slot = first, torch.where(key < n_experts, first[key] + rank, -1)
    place = torch.empty_like(slot).scatter_(0, sorted_, slot).int().view(experts.shape)
    source = torch.full((slots + 1,), -1, device=DEV, dtype=torch.long)
    source.scatter_(0, torch.where(slot < 0, slots, slot), torch.where(slot < 0, -1, sorted_))
    return dict(place=place, counts=counts.int(), starts=starts.int(), source=source[:slots].int())


def prepare(case, seed):
    gen = _generator(seed)

    def normal(shape, kind, scale):
        return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32).mul_(scale).to(TYPES[kind])

    n, s = case["tokens"], dict(case=case)
    if case["kind"] == "dropout":
        s.update(x=normal((n, case["width"]), case["type"], 1.0), seed=seed * 0x9E3779B9 + 1, call=seed % 1000)
        if case["add"]:
            s["held"] = normal((n, case["width"]), case["to"], 1.0)
        return s
    logits = _logits(case, gen)
    if case["kind"] == "gate":
        if case["masked"]:
            away = torch.rand(logits.shape, generator=gen, device=DEV) < case["masked"]
            logits = logits.masked_fill_(away, -math.inf)
        s["logits"] = logits.to(TYPES[case["type"]])
        if case["grad"]:
            s["experts"] = _top(s["logits"].float(), case["k"])[1].to(TYPES[case["index"]])
            s["g"] = normal((n, case["k"]), case["type"], 1.0)
        return s
    experts = _top(logits, case["k"])[1]
    del logits
    if case["kind"] == "sort":
        s["chosen"] = experts.to(TYPES[case["index"]])
        return s
    slots = _slots(case)
    if own:   # the order is made once for all calls on it
        from paper_2110_04478_amd import binding
        s["order"] = binding.themis_expert_sort(experts.int(), case["experts"], capacity=_capacity(case))
    else:
        s["order"] = _order(experts, case["experts"], _capacity(case), slots)
    if case["kind"] == "there":
        s["x"] = normal((slots if case["grad"] else n, case["width"]), case["type"], 1.0)
        return s
    s["y"] = normal((slots, case["width"]), case["type"], 1.0)
    s["weights"] = torch.softmax(torch.randn((n, case["k"]), generator=gen, device=DEV), -1).to(TYPES[case["weights"]])
    if case["grad"]:
        s["g"] = normal((n, case["width"]), case["to"], 1.0)
    elif case["add"]:
        s["held"] = normal((n, case["width"]), case["to"], 1.0)
    return s


def _run_own(s):
    from paper_2110_04478_amd import binding
    case = s["case"]
    if case["kind"] == "gate":
        chosen = case["over"] == "chosen"
        if case["grad"]:
            return binding.themis_expert_gate_grad(s["g"], s["logits"], s["experts"], renormalize=chosen,
                                                   out_dtype=TYPES[case["to"]])
        weights, experts = binding.themis_expert_gate(s["logits"], case["k"], renormalize=chosen,
                                                      out_dtype=TYPES[case["to"]], index_dtype=TYPES[case["index"]])
        return dict(weights=weights, experts=experts)
    if case["kind"] == "sort":
        order = binding.themis_expert_sort(s["chosen"], case["experts"], capacity=_capacity(case))
        return dict(place=order.place, counts=order.counts, starts=order.starts, source=order.source)
    if case["kind"] == "there":
        call = binding.themis_expert_combine if case["grad"] else binding.themis_expert_dispatch
        return call(s["x"], s["order"], out_dtype=TYPES[case["to"]])
    if case["kind"] == "back" and case["grad"]:
        rows, weights = binding.themis_expert_combine_grad(s["g"], s["y"], s["order"], s["weights"])
        return dict(rows=rows, weights=weights)
    if case["kind"] == "back":
        return binding.themis_expert_combine(s["y"], s["order"], s["weights"], out=s.get("held"),
                                             out_dtype=TYPES[case["to"]], accumulate=case["add"])
    return binding.themis_dropout(s["x"], case["p"], s["seed"], s["call"], add=s.get("held"),
                                  out_dtype=TYPES[case["to"]])


def _gate(s):
    case, logits = s["case"], s["logits"].float()
    values, experts = _top(logits, case["k"])
    if case["over"] == "chosen":
        e = torch.exp(values - values[:, :1])
        weights = e / e.sum(-1, keepdim=True)
    else:
        top = values[:, :1]
        weights = torch.exp(values - top) / torch.exp(logits - top).sum(-1, keepdim=True)
    weights = torch.where(experts < 0, 0.0, weights)
    return dict(weights=weights.to(TYPES[case["to"]]), experts=experts.to(TYPES[case["index"]]))


def _gate_grad(s):
    case, logits, g = s["case"], s["logits"].float(), s["g"].float()
    has, at = s["experts"] >= 0, s["experts"].long().clamp(min=0)
    values = torch.where(has, logits.gather(1, at), -math.inf)
    top = torch.where(has.any(-1, keepdim=True), values.amax(-1, keepdim=True), 0.0)
    e = torch.exp(values - top)
    if case["over"] == "chosen":
        total = e.sum(-1, keepdim=True)
        w = torch.where(total > 0, e / total, 0.0)
        grad = torch.zeros_like(logits)
    else:
        full = torch.exp(logits - top)
        total = full.sum(-1, keepdim=True)
        w = torch.where(total > 0, e / total, 0.0)
        grad = torch.where(total > 0, full / total, 0.0)
    dot = (w * g).sum(-1, keepdim=True)
    if case["over"] == "chosen":
        return grad.scatter_add_(1, at, w * (g - dot)).to(TYPES[case["to"]])
    return grad.mul_(-dot).scatter_add_(1, at, w * g).to(TYPES[case["to"]])


def _words(rows, blocks, seed, call):
    """Philox4x32-10 of Salmon, Moraes, Dror and Shaw (2011): four words for every counter
    (block of four columns, row, call), as whole numbers of 64 bits."""
    low = 0xFFFFFFFF
    c = [torch.arange(blocks, device=DEV).expand(rows, blocks), torch.arange(rows, device=DEV)[:, None].expand(rows, blocks),
         torch.full((), call & low, device=DEV), torch.full((), call >> 32 & low, device=DEV)]
    k0, k1 = seed & low, seed >> 32 & low
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32 & low) ^ c[1] ^ k0, b & low, (a >> 32 & low) ^ c[3] ^ k1, a & low]
        k0, k1 = k0 + 0x9E3779B9 & low, k1 + 0xBB67AE85 & low
    return c


def _kept(case, seed, call):
    words = torch.stack(_words(case["tokens"], -(-case["width"] // 4), seed, call), -1)
    return words.view(case["tokens"], -1)[:, :case["width"]] >= round(case["p"] * 2.0 ** 32)


def run(s):
    if own:
        return _run_own(s)
    case = s["case"]
    if case["kind"] == "gate":
        return _gate_grad(s) if case["grad"] else _gate(s)
    if case["kind"] == "sort":
        return _order(s["chosen"], case["experts"], _capacity(case), _slots(case))
    if case["kind"] == "dropout":
        x = torch.where(_kept(case, s["seed"], s["call"]), s["x"].float() * (1.0 / (1.0 - case["p"])), 0.0)
        if case["add"]:
            x = x.add_(s["held"])
        return x.to(TYPES[case["to"]])
    place, source, k = s["order"]["place"], s["order"]["source"], case["k"]
    if case["kind"] == "there" and not case["grad"]:
        rows = s["x"].float()[source.clamp(min=0) // k]
        return rows.masked_fill_((source < 0)[:, None], 0.0).to(TYPES[case["to"]])
    has, at = (place >= 0)[:, :, None], place.clamp(min=0)
    if case["kind"] == "there":
        return s["x"].float()[at].masked_fill_(~has, 0.0).sum(1).to(TYPES[case["to"]])
    weights = s["weights"].float()
    rows = s["y"].float()[at].masked_fill_(~has, 0.0)
    if not case["grad"]:
        out = rows.mul_(weights[:, :, None]).sum(1)
        return s["held"].copy_(out.add_(s["held"])) if case["add"] else out.to(TYPES[case["to"]])
    g = s["g"].float()
    grad = rows.mul_(g[:, None]).sum(-1)
    a = source.clamp(min=0)
    rows = g[a // k].mul_(weights.reshape(-1)[a][:, None]).masked_fill_((source < 0)[:, None], 0.0)
    return dict(rows=rows.to(TYPES[case["type"]]), weights=grad.to(TYPES[case["weights"]]))


def work(case):
    n = case["tokens"]
    if case["kind"] == "dropout":
        cells = n * case["width"]
        return {"bytes": cells * (SIZE[case["type"]] + SIZE[case["to"]] * (2 if case["add"] else 1)),
                "flops": cells * 2}
    pairs = n * case["k"]
    if case["kind"] == "gate":
        cells = n * case["experts"]
        if not case["grad"]:
            return {"bytes": cells * SIZE[case["type"]] + pairs * (SIZE[case["to"]] + SIZE[case["index"]]),
                    "flops": cells + 4 * pairs}
        read = pairs if case["over"] == "chosen" else cells
        return {"bytes": read * SIZE[case["type"]] + cells * SIZE[case["to"]] +
                pairs * (SIZE[case["type"]] + SIZE[case["index"]]), "flops": 4 * cells}
    slots = _slots(case)
    if case["kind"] == "sort":
        return {"bytes": pairs * (SIZE[case["index"]] + 4) + slots * 4 + case["experts"] * 8 + 4, "flops": pairs}
    kept, w = min(pairs, slots), case["width"]
    if case["kind"] == "there":
        if case["grad"]:
            return {"bytes": pairs * 4 + kept * w * SIZE[case["type"]] + n * w * SIZE[case["to"]], "flops": kept * w}
        return {"bytes": slots * 4 + n * w * SIZE[case["type"]] + slots * w * SIZE[case["to"]], "flops": 0}
    read = pairs * (4 + SIZE[case["weights"]]) + kept * w * SIZE[case["type"]]
    if not case["grad"]:
        return {"bytes": read + n * w * SIZE[case["to"]] * (2 if case["add"] else 1), "flops": 2 * kept * w}
    return {"bytes": read + n * w * SIZE[case["to"]] + slots * w * SIZE[case["type"]] + pairs * SIZE[case["weights"]],
            "flops": 3 * kept * w}


def _exact_words(rows, blocks, seed, call):
    """The same generator, its products in halves of 16 bits."""
    low = 0xFFFFFFFF

    def product(m, x):
        lo, hi = (m & 0xFFFF) * x, (m >> 16) * x          # below 2^48
        whole_low = ((hi & 0xFFFF) << 16) + (lo & low)
        return (hi >> 16) + (lo >> 32) + (whole_low >> 32), whole_low & low

    at = torch.arange(rows * blocks, device=DEV)
    word = [at % blocks, at // blocks, torch.zeros_like(at) + call % 2 ** 32, torch.zeros_like(at) + call // 2 ** 32]
    for r in range(10):
        key = ((seed % 2 ** 32 + r * 0x9E3779B9) % 2 ** 32, (seed // 2 ** 32 + r * 0xBB67AE85) % 2 ** 32)
        (high0, low0), (high1, low1) = product(0xD2511F53, word[0]), product(0xCD9E8D57, word[2])
        word = [high1 ^ word[1] ^ key[0], low1, high0 ^ word[3] ^ key[1], low0]
    return torch.stack(word, 1).view(rows, blocks * 4)


def exact(case, seed):
    """From the definitions in binary64."""
    if case["kind"] == "sort":
        return None   # whole numbers only
    s, n = prepare(case, seed), case["tokens"]
    if case["kind"] == "dropout":
        drop = _exact_words(n, (case["width"] + 3) // 4, s["seed"], s["call"])[:, :case["width"]] / 2.0 ** 32
        x = s["x"].double() / (1.0 - case["p"])
        x[drop < round(case["p"] * 2.0 ** 32) / 2.0 ** 32] = 0.0
        return x + s["held"].double() if case["add"] else x
    if case["kind"] == "gate":
        logits, k = s["logits"].double(), case["k"]
        if not case["grad"]:
            sorted_, _ = torch.sort(logits, dim=-1, descending=True)
            over = sorted_[:, :k] if case["over"] == "chosen" else logits
            weights = torch.exp(sorted_[:, :k] - torch.logsumexp(over, -1, keepdim=True))
            return dict(weights=torch.nan_to_num(weights, nan=0.0), experts=None)
        # d weights[j] / d logits[e] = weights[j] * ((e is j's) - p[e]), p the softmax behind the weights
        hot = (s["experts"].long()[:, :, None] == torch.arange(case["experts"], device=DEV)).double()
        if case["over"] == "chosen":
            logits = torch.where(hot.sum(1) > 0, logits, -math.inf)
        p = torch.nan_to_num(torch.softmax(logits, -1), nan=0.0)
        pull = ((hot * p[:, None]).sum(-1) * s["g"].double())[:, :, None]
        return (pull * (hot - p[:, None])).sum(1)
    order = s["order"]
    k, slots = case["k"], _slots(case)
    source = (order["source"] if isinstance(order, dict) else order.source).long()
    slot = (source >= 0).nonzero().view(-1)
    pair = source[slot]
    token = pair // k
    if case["kind"] == "there":
        x = s["x"].double()
        if case["grad"]:
            return torch.zeros((n, case["width"]), dtype=torch.float64, device=DEV).index_add_(0, token, x[slot])
        return torch.zeros((slots, case["width"]), dtype=torch.float64, device=DEV).index_copy_(0, slot, x[token])
    weights = s["weights"].double().view(-1)[pair][:, None]
    if not case["grad"]:
        out = s["held"].double() if case["add"] else torch.zeros((n, case["width"]), dtype=torch.float64, device=DEV)
        return out.index_add_(0, token, s["y"].double()[slot].mul_(weights))
    g = s["g"].double()[token]
    grad = torch.zeros(n * k, dtype=torch.float64, device=DEV)
    grad[pair] = (g * s["y"].double()[slot]).sum(-1)
    rows = torch.zeros((slots, case["width"]), dtype=torch.float64, device=DEV)
    rows[slot] = g.mul_(weights)
    return dict(rows=rows, weights=grad.view(n, k))
