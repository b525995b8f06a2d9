"""Answering from retained caches: one image request, compressed as it is prefilled, and a few short text prompts, packed,
share a pool of pages and decode together.

    python examples/serve.py [--steps 16] [--page-format int8]

Weights are random and there is no vocabulary: a "model" here is, per layer, three projections, attention and an output
projection with a residual.  What matters is the order of the calls:

  prefill   Kvc.prefill_chunk            block by block, the cache of every layer held to a budget
            Pool.write                   the retained cache of every layer into the pool's pages (8 bits if asked for)
            Pool.prompt + Pool.write     all short prompts at once, in one launch per layer
  decode    Pool.decode                  one token for every sequence: its row is appended and attended to in one launch per layer
            (the step is captured once as a CUDA graph; lengths live on the device and grow by themselves)
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2604_16734_b200.binding import Kvc  # noqa: E402
from paper_2604_16734_b200.pool import Pool  # noqa: E402


class Toy:
    """Random weights of a decoder with grouped heads; ``mix`` is what stands between two layers' attention calls."""

    def __init__(self, layers=3, hq=8, hkv=2, d=64, width=256, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.layers, self.hq, self.hkv, self.d, self.width = layers, hq, hkv, d, width
        new = lambda a, b: (torch.randn(a, b, generator=g, device="cuda") * a ** -0.5).bfloat16()  # noqa: E731
        self.qkv = [new(width, (hq + 2 * hkv) * d) for _ in range(layers)]
        self.o = [new(hq * d, width) for _ in range(layers)]

    def project(self, layer, x):
        """q, k, v as the fused projection leaves them: heads of one row of numbers per token."""
        n = x.shape[0]
        x = torch.nn.functional.rms_norm(x, (self.width,))
        return (x @ self.qkv[layer]).view(n, self.hq + 2 * self.hkv, self.d).split([self.hq, self.hkv, self.hkv], 1)

    def mix(self, layer, x, attended):
        return x + attended.reshape(x.shape[0], -1) @ self.o[layer]


def serve(image_tokens=300, budget=128, chunk=64, prompts=(23, 1, 150), steps=16, page_format="plain", page_size=16, seed=0,
          model=None, trace=None):
    """Runs the requests; returns the last hidden states [steps][sequences][width].  ``trace`` collects what each decode
    call was given and gave."""
    m = model or Toy(seed=seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    tokens = lambda n: torch.randn(n, m.width, generator=g, device="cuda").bfloat16()  # noqa: E731
    n_seqs = 1 + len(prompts)
    per_seq = -(-(max(budget, *prompts) + steps) // page_size)
    pool = Pool(m.hq, m.hkv, m.d, torch.bfloat16, n_pages=n_seqs * per_seq, page_size=page_size, page_format=page_format, n_layers=m.layers,
                max_seqs=n_seqs)
    table = torch.arange(n_seqs * per_seq, dtype=torch.int32, device="cuda").view(n_seqs, per_seq)
    last = torch.empty(n_seqs, m.width, dtype=torch.bfloat16, device="cuda")

    # the image request: every block through every layer, the caches never longer than the budget
    kvc = Kvc(m.layers, m.hq, m.hkv, m.d, torch.bfloat16, budget, chunk)
    image = tokens(image_tokens)
    for first in range(0, image_tokens, chunk):
        x = image[first:first + chunk]
        for layer in range(m.layers):
            q, k, v = (t.contiguous() for t in m.project(layer, x))
            x = m.mix(layer, x, kvc.prefill_chunk(layer, q, k, v, first))
    last[0] = x[-1]
    for layer in range(m.layers):
        K, V, _, n = kvc.cache_view(layer)                        # [kv-head][row][d], n rows retained
        pool.write(layer, K[:, :n].transpose(0, 1), V[:, :n].transpose(0, 1), pool.slots(table[0], n))
    lens = [n, *prompts]

    # the text prompts: packed, uncompressed
    plan = pool.plan(prompts)
    slots = torch.cat([pool.slots(table[i + 1], n) for i, n in enumerate(prompts)])
    x = tokens(sum(prompts))
    for layer in range(m.layers):
        q, k, v = m.project(layer, x)
        attended, _ = pool.prompt(q, k, v, plan)
        pool.write(layer, k, v, slots)
        x = m.mix(layer, x, attended)
    ends = torch.tensor(prompts, device="cuda").cumsum(0) - 1
    last[1:] = x[ends]

    # one token for everybody, again and again
    lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
    states = []

    def step():
        x = last
        for layer in range(m.layers):
            q, k, v = m.project(layer, x)
            attended, lse = pool.decode(layer, q, table, lens, k, v)
            if trace is not None:
                trace.append((layer, q, k, v, attended, lse))
            x = m.mix(layer, x, attended)
        last.copy_(x)
        lens.add_(1)

    start = last.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                                 # once outside the capture: it also writes row lens[i], which the first
        step()                                                    # replay writes again
    torch.cuda.current_stream().wait_stream(side)
    lens.sub_(1)
    last.copy_(start)
    if trace is not None:
        trace.clear()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(steps):
        graph.replay()
        states.append(last.clone())
    assert pool.status() == 0 and kvc.status() == 0
    return torch.stack(states), pool, table, lens


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=16)
    ap.add_argument("--page-format", choices=["plain", "int8"], default="plain")
    a = ap.parse_args()
    states, pool, _, lens = serve(steps=a.steps, page_format=a.page_format)
    print(f"{a.steps} steps for {states.shape[1]} sequences, lengths now {lens.tolist()}, {pool.launch_count()} launches of the pool's calls")
    print("last hidden states, norms:", [round(x, 2) for x in states[-1].float().norm(dim=-1).tolist()])


if __name__ == "__main__":
    main()
