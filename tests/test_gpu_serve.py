"""The example that runs prefill, hand-over, packed prompts and decode together, held to the definitions in 64 bits."""
import math
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("page_format", ["plain", "int8"])
def test_example_answers_from_the_caches_it_holds(page_format):
    import serve
    steps, prompts, budget = 5, (23, 1, 150), 128
    trace = []
    states, pool, table, lens = serve.serve(steps=steps, prompts=prompts, budget=budget, page_format=page_format, trace=trace)
    assert lens.tolist() == [budget + steps, *(n + steps for n in prompts)] and bool(torch.isfinite(states).all())
    # the last replay's calls against what the pages hold now: rows [0, lens) of every sequence, the step's own token last
    for layer, q, k, v, attended, lse in trace:
        for i, n in enumerate(lens.tolist()):
            K, V = pool.read(layer, pool.slots(table[i], n))
            if page_format == "plain":
                assert torch.equal(K[-1], k[i]) and torch.equal(V[-1], v[i])
            group = q.shape[1] // K.shape[1]
            K, V = (x.double().repeat_interleave(group, 1) for x in (K, V))
            z = torch.einsum("hd,nhd->hn", q[i].double(), K) / math.sqrt(q.shape[2])
            want = torch.einsum("hn,nhd->hd", torch.softmax(z, -1), V)
            # (8-bit rows are read back rounded to bf16, 2^-9 of a value: keys move a score by 2^-9 of its terms' sum)
            off = 2e-2 if page_format == "plain" else 2e-2 + 2.0 ** -8 * V.abs().max().item()
            assert (attended[i].double() - want).abs().max() <= off
            assert (lse[i].double() - torch.logsumexp(z, -1)).abs().max() <= (2e-3 if page_format == "plain" else 2e-2)


def test_example_in_eight_bits_stays_near_the_plain_one():
    import serve
    a, *_ = serve.serve(steps=3, page_format="plain")
    b, *_ = serve.serve(steps=3, page_format="int8")
    # rows of normal numbers in steps of max / 127 (max of 64: about 2.5) are off by 2.5 / 127 / sqrt(12) = 0.6 % of their size
    assert (a[0].double() - b[0].double()).norm() / a[0].double().norm() < 2e-2
