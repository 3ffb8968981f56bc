"""A training iteration's gradients, and how long a network takes to sum them.

A small next-token model with a tied token table is trained for a few steps.  Every step looks
tokens up, adds the table's gradient to the output projection's, lays all gradients into the flat
buckets that the ranks' All-Reduces carry, and clips what comes back by the norm of the sum; the
parameters are updated from the buckets.  The sizes of the buckets are then a trace for the evaluator: it
plans and simulates the iteration's All-Reduces on the six platforms of the paper's Table 2.

With experts the feed-forward layer is one of experts in buffers of a fixed capacity, whose gradients go into the
same buckets; with dropout what the layer adds to the residual is dropped by a counter.

    python examples/training_iteration.py [steps [experts [dropout]]]
"""
import math
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2110_04478_amd import binding, layers, workloads  # noqa: E402
from paper_2110_04478_amd.gradients import GradientBuckets, embedding  # noqa: E402

PAD = 0
CHOSEN, CAPACITY = 2, 1.5   # experts of a token; an expert's buffer over the mean load
SEED = 11


def model(vocab, width, device, seed, experts=0):
    g = torch.Generator().manual_seed(seed)

    def weight(*shape):   # (by what a sum goes over: a row, or of an expert's matrix, which stands to the right, a column)
        terms = shape[-1] if len(shape) == 2 else shape[-2]
        return torch.nn.Parameter((torch.randn(shape, generator=g) / math.sqrt(terms)).to(device))

    if experts:
        return dict(table=weight(vocab, width), router=weight(experts, width), up=weight(experts, width, 4 * width),
                    down=weight(experts, 4 * width, width))
    return dict(table=weight(vocab, width), up=weight(4 * width, width), down=weight(width, 4 * width))


def feed_forward(p, x):
    if "router" not in p:
        return torch.relu(x @ p["up"].t()) @ p["down"].t()
    n_experts, width = p["up"].shape[:2]
    k = min(CHOSEN, n_experts)
    capacity = math.ceil(CAPACITY * k * x[..., 0].numel() / n_experts)
    weights, chosen = layers.gate(x @ p["router"].t(), k)
    order = layers.sort(chosen, n_experts, capacity)
    rows = layers.dispatch(x, order).view(n_experts, capacity, width)
    rows = torch.bmm(torch.relu(torch.bmm(rows, p["up"])), p["down"])
    return layers.combine(rows.view(order.slots, width), order, weights)


def loss_of(p, tokens, dropout=0.0, step=0):
    """Next-token loss; padding is looked up but has no gradient and is not predicted."""
    width = p["table"].shape[1]
    x = embedding(p["table"], tokens[:, :-1], math.sqrt(width), ignored=PAD, into=p["table"].grad)
    y = feed_forward(p, x)
    x = layers.dropout(y, dropout, SEED, step, add=x) if dropout else x + y
    x = x / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt()
    logits = x @ p["table"].t()
    return torch.nn.functional.cross_entropy(logits.flatten(0, 1), tokens[:, 1:].flatten(), ignore_index=PAD)


def batch_of(vocab, batch, length, device, seed):
    """Sequences that count upwards by three, and end in padding."""
    r = np.random.default_rng(seed)
    tokens = (r.integers(1, vocab, (batch, 1)) + 3 * np.arange(length)) % (vocab - 1) + 1
    tokens[np.arange(length) >= r.integers(length // 2, length + 1, (batch, 1))] = PAD
    return torch.from_numpy(tokens).to(device)


def iteration_times(sizes, chunks=64):
    """Completion times of the iteration's All-Reduces on the Table 2 platforms under the three
    schedulers -> f64[3, 6] (baseline, Themis+FIFO, Themis+SCF)."""
    times = []
    for inter, intra in ((workloads.INTER_BASELINE, workloads.INTRA_FIFO),
                         (workloads.INTER_THEMIS, workloads.INTRA_FIFO),
                         (workloads.INTER_THEMIS, workloads.INTRA_SCF)):
        b = workloads.table2(sizes_bytes=(1.0,), chunks=chunks, inter=inter, intra=intra, with_latency=False)
        b.max_coll = len(sizes)
        b.n_coll = np.full(b.n, len(sizes), dtype=np.uint32)
        b.coll_size = np.ascontiguousarray(np.repeat(np.asarray(sizes)[:, None], b.n, axis=1))
        d = binding.to_device(b)
        orders, _ = binding.themis_plan_batch(d)
        ws = binding.alloc_workspace(binding.themis_workspace_bytes(d.n, d.max_chunks, d.max_coll))
        t, _, _ = binding.themis_simulate_batch(d, orders, workspace=ws, want_queue_order=False)
        times.append(t.cpu().numpy())
    return np.stack(times)


def main(steps=40, vocab=2000, width=256, batch=16, length=128, rate=2.0, max_norm=1.0, device="cuda:0",
         all_reduce=lambda buckets: None, experts=0, dropout=0.0):
    """all_reduce: sums the buckets over the ranks, in place (one rank: they are the sum)."""
    p = model(vocab, width, device, 1, experts)
    buckets = GradientBuckets(p.values(), bucket_bytes=1 << 20)
    losses, norms = [], []
    for step in range(steps):
        buckets.zero()
        loss = loss_of(p, batch_of(vocab, batch, length, device, step), dropout, step)
        loss.backward()
        buckets.fill()
        all_reduce(buckets.buckets)
        total, _ = buckets.clip_summed(max_norm)
        with torch.no_grad():
            for q in buckets.params:
                q.sub_(buckets.views[q], alpha=rate)
        losses.append(loss.detach())
        norms.append(total[0])
    return dict(losses=torch.stack(losses).tolist(), norms=torch.stack(norms).tolist(),
                sizes=buckets.sizes(), times=iteration_times(buckets.sizes()))


if __name__ == "__main__":
    got = main(int(sys.argv[1]) if len(sys.argv) > 1 else 40, experts=int(sys.argv[2]) if len(sys.argv) > 2 else 0,
               dropout=float(sys.argv[3]) if len(sys.argv) > 3 else 0.0)
    print("loss %.3f -> %.3f, norm of the gradients %.3f -> %.3f" %
          (got["losses"][0], got["losses"][-1], got["norms"][0], got["norms"][-1]))
    print("buckets of the iteration, bytes: %s" % ", ".join("%d" % s for s in got["sizes"]))
    for name, t in zip((t[0] for t in workloads.TABLE2), got["times"].T):
        print("%-22s baseline %.1f us  Themis+FIFO %.1f us  Themis+SCF %.1f us" % (name, *(t * 1e6)))
