"""One layer's decode steps with everything this package has for them, as a serving loop runs them:

    the predictor names the experts before attention runs (to be prefetched),
    the new token's keys and values are appended to the paged cache,
    attention runs over the cache and adds up every position's weight,
    the expert layer runs on the router's own selection,
    the prediction is scored against it,
    and when the cache is full, the positions of least weight are evicted into free pages.

Synthetic weights and states of a model's shape; prints the prefetch lists' sizes and the predictor's hit rate.

    python examples/decode_step.py [--steps N]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2511_10676_amd import binding as B  # noqa: E402


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=48)
    steps = ap.parse_args().steps
    seqs, Hq, Hkv, D, page = 6, 32, 4, 128, 16                 # sequences, heads, head width, positions per page
    d, r, E, k, k_over, f = 2048, 2048, 128, 8, 12, 768        # hidden size, predictor width, experts, selected, predicted, expert width
    budget, recent, prompt = 256, 32, 240
    wide = -(-(budget + 64) // page)                           # pages of a sequence: the budget and room to grow
    g = torch.Generator(device="cuda").manual_seed(7)

    def randn(*shape, std=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * std).to(torch.bfloat16)

    # weights: the router, a predictor that has learned most of it (two linear maps whose product is close to the router's),
    # the experts, and the projections around attention
    W1, W2 = randn(r, d, std=d ** -0.5), randn(E, r, std=r ** -0.5)
    Wg = (W2.float() @ W1.float() + 0.1 * torch.randn((E, d), generator=g, device="cuda") * d ** -0.5).to(torch.bfloat16)
    W13, W_down = randn(E, 2 * f, d, std=d ** -0.5), randn(E, d, f, std=f ** -0.5)
    Wqkv, Wo = randn((Hq + 2 * Hkv) * D, d, std=d ** -0.5), randn(d, Hq * D, std=0.1 * (Hq * D) ** -0.5)

    # the cache: two sets of pages per sequence, one in use, one free to evict into
    pools = torch.zeros((2, 2 * seqs * wide, Hkv, page, D), dtype=torch.bfloat16, device="cuda")
    k_pages, v_pages = pools[0], pools[1]
    tables = torch.randperm(2 * seqs * wide, generator=g, device="cuda").to(torch.int32).view(2, seqs, wide).contiguous()
    table, free = tables[0], tables[1]
    capacity = wide * page
    mass = torch.zeros((seqs, Hkv, capacity), device="cuda")
    lengths = torch.full((seqs,), prompt, dtype=torch.int32, device="cuda")
    at = torch.arange(prompt, dtype=torch.int32, device="cuda").repeat(seqs)
    who = torch.arange(seqs, dtype=torch.int32, device="cuda").repeat_interleave(prompt)
    B.cache_append(randn(seqs * prompt, Hkv, D), randn(seqs * prompt, Hkv, D), k_pages, v_pages, table, at, sequences=who, mass=mass)

    x = randn(seqs, d)
    counters = torch.zeros((1, 4), dtype=torch.int64, device="cuda")
    longest = prompt
    for step in range(steps):
        norm = (x.float() * x.float().square().mean(dim=1, keepdim=True).rsqrt()).to(torch.bfloat16)
        predicted = B.predict(norm, W1, W2, k_over)             # before attention: what to prefetch
        lists = B.group_by_expert(predicted.idx, E)
        qkv = norm @ Wqkv.t()
        new_k = qkv[:, Hq * D:(Hq + Hkv) * D].unflatten(1, (Hkv, D))
        new_v = qkv[:, (Hq + Hkv) * D:].unflatten(1, (Hkv, D))
        B.cache_append(new_k, new_v, k_pages, v_pages, table, lengths, mass=mass)
        lengths, longest = lengths + 1, longest + 1
        out = B.attend(qkv[:, :Hq * D].unflatten(1, (Hq, D)), k_pages, v_pages, table, lengths, mass=mass, max_len=longest).out
        x = x + out.flatten(1) @ Wo.t()
        norm = (x.float() * x.float().square().mean(dim=1, keepdim=True).rsqrt()).to(torch.bfloat16)
        layer = B.moe_layer(norm, Wg, W13, W_down, k, prob="softmax_topk", residual=x)
        x = layer.y
        counters += B.score(predicted.idx, layer.idx[None], E)
        if longest == capacity:                                 # full: cut every sequence to the budget, swap the page sets
            cut = B.cache_evict(k_pages, v_pages, table, lengths, mass, free, budget, recent, max_len=longest)
            table, free, mass, lengths, longest = free, table, cut.mass, cut.lengths, budget
            print(f"step {step}: evicted to {budget} positions")
    torch.cuda.synchronize()
    hit = counters[0, 1].item() / (steps * seqs * k)
    print(f"{steps} steps of {seqs} sequences: last prefetch list {int(lists.n_active[0])} experts, "
          f"{100 * hit:.1f} % of the router's experts were among the {k_over} predicted, states finite: {bool(x.isfinite().all())}")
    return hit


if __name__ == "__main__":
    main()
