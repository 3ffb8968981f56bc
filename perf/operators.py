"""Workloads of the gradient operators: what a rank computes on the gradients of an
iteration before the modelled collective carries them.

Every case is one call of a public entry point on tensors that are already in HBM.
Four kinds:

  lookup  themis_embedding_lookup: rows of a token table, scaled
  grad    themis_embedding_grad: the table's gradient, written whole or added to one
  norm    themis_gradient_norm: the norm of every tensor and of all of them
  clip    themis_gradient_clip: the same, and the clipped gradients in one flat bucket

Fields of a case:
  tokens, width, vocab   tokens looked up, elements of a row, rows of the table
  type, to               element types of what is read and of what is written
  index                  type of the token numbers
  scale                  factor on the rows (and on their gradient)
  hot      grad: share of the tokens that are one and the same (a separator, padding that is
           trained); the others follow the usual law of words, probability ~ 1 / (rank + 1)
  ignored  grad: share of the tokens that have no gradient (padding)
  add      grad: added to a table that holds a gradient already (a tied output
           projection, or the micro-batches before)
  layers   norm, clip: transformer blocks of `width` whose gradients are the list, behind
           a table of `vocab` rows; type "mixed": matrices in bf16, vectors in f32
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16,
         "i32": torch.int32, "i64": torch.int64}
MAX_NORM = 1.0


def listed():
    return [
        # the smallest call: one token of a decoding step
        dict(name="next token", kind="lookup", tokens=1, width=4096, vocab=32768, type="bf16",
             to="bf16", index="i64", scale=1.0),
        # a prompt on odd sizes, master weights in binary32, activations in bf16
        dict(name="odd prompt", kind="lookup", tokens=8191, width=1001, vocab=50003, type="f32",
             to="bf16", index="i64", scale=31.6),
        # the input of a training step: 16 sequences of 4096 tokens
        dict(name="training input", kind="lookup", tokens=65536, width=4096, vocab=131072,
             type="bf16", to="bf16", index="i64", scale=64.0),
        # one short sequence, added to the gradient of the tied output projection
        dict(name="short sequence, tied", kind="grad", tokens=512, width=1024, vocab=32768,
             type="bf16", to="f32", index="i64", scale=32.0, hot=0.0, ignored=0.0, add=True),
        # the table's gradient of a training step, written whole
        dict(name="training gradient", kind="grad", tokens=16384, width=4096, vocab=131072,
             type="bf16", to="bf16", index="i64", scale=64.0, hot=0.0, ignored=0.1, add=False),
        # many short sequences: one separator makes up half of the tokens; odd sizes
        dict(name="half one token", kind="grad", tokens=65537, width=1000, vocab=50003, type="f16",
             to="f32", index="i32", scale=1.0, hot=0.5, ignored=0.0, add=False),
        # a large micro-batch on a tied table
        dict(name="micro-batch, tied", kind="grad", tokens=131072, width=2048, vocab=65536,
             type="bf16", to="f32", index="i64", scale=1.0, hot=0.05, ignored=0.0, add=True),
        # the list of a small model: many tiny tensors, latency
        dict(name="norm of a small model", kind="norm", width=96, layers=2, vocab=1024, type="f32"),
        # a rank's gradients of a large model
        dict(name="norm of a large model", kind="norm", width=4096, layers=8, vocab=32768,
             type="bf16"),
        # the small model again, clipped into its bucket; two types, tensors at odd places
        dict(name="clip of a small model", kind="clip", width=97, layers=2, vocab=1023,
             type="mixed", to="f32"),
        # an ordinary model: about what the last cache level holds
        dict(name="clip of an ordinary model", kind="clip", width=1024, layers=8, vocab=32768,
             type="bf16", to="bf16"),
        # the largest: a rank's binary32 gradients into the collective's bf16 bucket
        dict(name="clip of a large model", kind="clip", width=4096, layers=4, vocab=65536,
             type="f32", to="bf16"),
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
    return n | 1 if n | 1 <= hi else (n - 2) | 1


def draw(rng):
    kind = rng.choices(("lookup", "grad", "norm", "clip"), (25, 35, 15, 25))[0]
    case = dict(kind=kind)
    if kind in ("lookup", "grad"):
        width = _size(rng, 32, 8192)
        vocab = _size(rng, 256, min(262144, (1 << 29) // width))
        tokens = _size(rng, 1, min(131072, (1 << 28) // width))
        kinds = rng.choice((("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("f32", "bf16"),
                            ("bf16", "f32"), ("f16", "f32")))
        case.update(tokens=tokens, width=width, vocab=vocab, type=kinds[0], to=kinds[1],
                    index=rng.choice(("i64", "i64", "i32")),
                    scale=rng.choice((1.0, round(math.sqrt(width), 3))))
        if kind == "grad":
            case.update(hot=rng.choice((0.0, 0.0, 0.05, 0.3, 0.9)),
                        ignored=rng.choice((0.0, 0.0, 0.1, 0.6)), add=rng.random() < 0.4)
    else:
        width = _size(rng, 16, 4096)
        vocab = _size(rng, 64, min(131072, (1 << 29) // width))
        most = ((1 << 30) - vocab * width) // (12 * width * width + 13 * width)
        case.update(width=width, layers=_log_int(rng, 1, max(1, min(48, most))), vocab=vocab,
                    type=rng.choice(("f32", "bf16", "bf16", "f16", "mixed")))
        if kind == "clip":
            case["to"] = rng.choice(("f32", "bf16", "bf16", "f16"))
    return case


def _shapes(case):
    """The list of a transformer's gradients: a table, blocks of two norms, four projections
    and two feed-forward matrices with their biases, and a last norm."""
    w = case["width"]
    block = [(w,), (w, w), (w, w), (w, w), (w, w), (w,), (4 * w, w), (4 * w,), (w, 4 * w), (w,)]
    return [(case["vocab"], w)] + block * case["layers"] + [(w,)]


def _types(case):
    kinds = {"f32": (torch.float32,) * 2, "bf16": (torch.bfloat16,) * 2, "f16": (torch.float16,) * 2,
             "mixed": (torch.bfloat16, torch.float32)}[case["type"]]
    return [kinds[len(s) == 1] for s in _shapes(case)]


def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _ids(case, gen):
    """Token numbers: rank r with probability ~ 1 / (r + 1); a share is one token, a share has none."""
    n, vocab = case["tokens"], case["vocab"]
    u = torch.rand(n, generator=gen, device=DEV, dtype=torch.float64)
    ids = (torch.exp(u * math.log(vocab + 1.0)).long() - 1).clamp_(0, vocab - 1)
    pick = torch.rand(n, generator=gen, device=DEV)
    hot, ignored = case.get("hot", 0.0), case.get("ignored", 0.0)
    ids = torch.where(pick < hot, vocab // 3, ids)
    ids = torch.where(pick >= 1.0 - ignored * (1.0 - hot), _padding(case), ids)
    return ids.to(TYPES[case["index"]])


def _padding(case):
    """The token number that has no gradient."""
    return case["vocab"] - 1 if case.get("ignored", 0.0) > 0 else -1


def prepare(case, seed):
    gen = _generator(seed)

    def normal(shape, kind, scale):
        return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32).mul_(scale).to(kind)

    if case["kind"] == "lookup":
        return dict(case=case, ids=_ids(case, gen),
                    table=normal((case["vocab"], case["width"]), TYPES[case["type"]], 0.02))
    if case["kind"] == "grad":
        s = dict(case=case, ids=_ids(case, gen),
                 g=normal((case["tokens"], case["width"]), TYPES[case["type"]], 0.01))
        if case["add"]:
            s["held"] = normal((case["vocab"], case["width"]), TYPES[case["to"]], 0.01)
        return s
    # scales of the tensors differ, as they do between layers, vectors and matrices
    scales = np.random.default_rng(seed).uniform(-9.0, -4.0, len(_shapes(case)))
    grads = [normal(shape, kind, math.exp(e))
             for shape, kind, e in zip(_shapes(case), _types(case), scales)]
    s = dict(case=case, grads=grads)
    if case["kind"] == "clip":   # the bucket that the collective carries: tensors end to end
        s["bucket"] = torch.empty(sum(g.numel() for g in grads), dtype=TYPES[case["to"]], device=DEV)
    if own:   # laid out once, as long as the gradients stay where they are
        from paper_2110_04478_amd import binding
        out = None
        if case["kind"] == "clip":
            parts = s["bucket"].split([g.numel() for g in grads])
            out = [p.view(g.shape) for p, g in zip(parts, grads)]
        s["plan"] = binding.themis_gradient_plan(grads, out)
    return s


def _run_own(s):
    from paper_2110_04478_amd import binding
    case = s["case"]
    if case["kind"] == "lookup":
        return binding.themis_embedding_lookup(s["table"], s["ids"], case["scale"],
                                               out_dtype=TYPES[case["to"]])
    if case["kind"] == "grad":
        return binding.themis_embedding_grad(s["g"], s["ids"], case["vocab"], case["scale"],
                                             ignored=_padding(case), out=s.get("held"),
                                             out_dtype=TYPES[case["to"]], accumulate=case["add"])
    if case["kind"] == "norm":
        total, norms = binding.themis_gradient_norm(s["plan"])
        return dict(total=total, norms=norms)
    total, norms = binding.themis_gradient_clip(s["plan"], MAX_NORM)
    return dict(total=total, norms=norms, bucket=s["bucket"])


def run(s):
    if own:
        return _run_own(s)
    case = s["case"]
    if case["kind"] == "lookup":
        return (s["table"][s["ids"]].float() * case["scale"]).to(TYPES[case["to"]])
    if case["kind"] == "grad":
        g = s["g"].float()
        if case["ignored"]:
            g = g * (s["ids"] != _padding(case))[:, None]
        total = torch.zeros((case["vocab"], case["width"]), dtype=torch.float32, device=DEV)
        total.index_add_(0, s["ids"], g).mul_(case["scale"])
        if case["add"]:
            return s["held"].copy_(total.add_(s["held"]))
        return total.to(TYPES[case["to"]])
    squares = torch.stack([g.float().square().sum() for g in s["grads"]])
    total = squares.sum().sqrt()
    if case["kind"] == "norm":
        return dict(total=total[None], norms=squares.sqrt())
    factor = (MAX_NORM / total).clamp(max=1.0)
    bucket = torch.cat([(g.float() * factor).to(TYPES[case["to"]]).view(-1) for g in s["grads"]])
    return dict(total=torch.stack([total, factor]), norms=squares.sqrt(), bucket=bucket)


def _probabilities(case):
    """Probability of every token number, and that of one without a gradient."""
    r = np.arange(case["vocab"], dtype=np.float64)
    p = np.log((r + 2.0) / (r + 1.0)) / math.log(case["vocab"] + 1.0)
    hot, ignored = case.get("hot", 0.0), case.get("ignored", 0.0) * (1.0 - case.get("hot", 0.0))
    p *= 1.0 - hot - ignored
    p[case["vocab"] // 3] += hot
    return p, ignored


def work(case):
    size = {"f32": 4, "bf16": 2, "f16": 2, "i32": 4, "i64": 8}
    if case["kind"] in ("lookup", "grad"):
        p, ignored = _probabilities(case)
        rows = float(-np.expm1(case["tokens"] * np.log1p(-np.minimum(p, 1.0 - 1e-12))).sum())
        cells, index = case["tokens"] * case["width"], case["tokens"] * size[case["index"]]
        if case["kind"] == "lookup":
            return {"bytes": index + rows * case["width"] * size[case["type"]] +
                    cells * size[case["to"]], "flops": cells}
        cells *= 1.0 - ignored
        written = 2 * rows if case["add"] else case["vocab"]
        return {"bytes": index + cells * size[case["type"]] +
                written * case["width"] * size[case["to"]], "flops": cells}
    counts = [math.prod(s) for s in _shapes(case)]
    read = sum(n * t.itemsize for n, t in zip(counts, _types(case))) + 4 * len(counts)
    if case["kind"] == "norm":
        return {"bytes": read, "flops": 2 * sum(counts)}
    return {"bytes": read + sum(counts) * size[case["to"]], "flops": 3 * sum(counts)}


def exact(case, seed):
    """From the definitions in binary64."""
    s = prepare(case, seed)
    if case["kind"] == "lookup":
        return torch.index_select(s["table"], 0, s["ids"].long()).double().mul_(case["scale"])
    if case["kind"] == "grad":
        ids = s["ids"].long()
        has = (ids != _padding(case)).nonzero().view(-1)
        total = torch.zeros((case["vocab"], case["width"]), dtype=torch.float64, device=DEV)
        total.index_put_((ids[has],), s["g"][has].double() * case["scale"], accumulate=True)
        return total.add_(s["held"]) if case["add"] else total
    norms = torch.stack([torch.linalg.vector_norm(g, dtype=torch.float64) for g in s["grads"]])
    total = torch.linalg.vector_norm(norms)
    if case["kind"] == "norm":
        return dict(total=total[None], norms=norms)
    factor = torch.minimum(MAX_NORM / total, torch.ones_like(total))
    return dict(total=torch.stack([total, factor]), norms=norms,
                bucket=torch.cat([g.reshape(-1).double() * factor for g in s["grads"]]))
