"""A decoder that serves a few requests: the block tables, the 4-bit KV cache, attention over it and the verification
of drafted tokens, called in turn as a serving loop calls them.

    python examples/decode_loop.py [--drafts 3]

The model is the smallest that has a cache: one attention layer whose queries, keys and values are rows of tables (one
row a token), and a projection to the vocabulary; weights are random.  The drafter guesses the token that last followed
the same token.  A step feeds every live request its last token and the drafts behind it, and keeps what the model
accepts; the rejected tokens' places in the cache are used again by the next step.
"""
from __future__ import annotations

import argparse
import os
import sys
from dataclasses import dataclass

if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_2609_15359_amd as maps


@dataclass
class Model:
    """One attention layer of a vocabulary's tables."""
    q: torch.Tensor         # [V, q_heads, dim]
    k: torch.Tensor         # [V, heads, dim]
    v: torch.Tensor
    proj: torch.Tensor      # [q_heads * dim, V] float32
    temperature: float

    @classmethod
    def random(cls, vocab=500, heads=2, group=4, dim=64, temperature=1.0, dtype=torch.bfloat16, device="cuda", seed=0):
        g = torch.Generator().manual_seed(seed)

        def table(*shape):
            return torch.randn(shape, generator=g)
        return cls(q=(2 * table(vocab, heads * group, dim)).to(device, dtype), k=table(vocab, heads, dim).to(device, dtype),
                   v=table(vocab, heads, dim).to(device, dtype), proj=table(heads * group * dim, vocab).to(device),
                   temperature=temperature)

    @property
    def scale(self) -> float:
        return self.k.shape[2] ** -0.5

    def probabilities(self, out):
        return torch.softmax(out.flatten(1).float() @ self.proj / self.temperature, -1)


def serve(model: Model, prompts, new_tokens: int, drafts: int, cache_bytes: int, block_size: int = 16, seed: int = 0):
    """Answers every prompt (a list of lists of tokens) with new_tokens tokens; returns the answers and the number of
    steps that it took.  cache_bytes is the decoder's KV memory."""
    dev = model.q.device
    B, K, V = len(prompts), drafts, model.q.shape[0]
    heads, dim = model.k.shape[1:]
    g = torch.Generator(device=dev).manual_seed(seed)

    # the decoder's capacity as placement counts it, and its blocks
    per_token = maps.KVCache.bytes_per_token(heads, dim)
    capacity = maps.capacity_tokens(torch.tensor([cache_bytes], dtype=torch.int64, device=dev), per_token)
    blocks = int(capacity.item()) // block_size
    longest = max(map(len, prompts)) + new_tokens + K
    if sum(-(-(len(p) + new_tokens + K) // block_size) for p in prompts) > blocks:
        raise ValueError("the cache is too small for these requests")
    cache = maps.KVCache.empty(blocks, heads, dim, block_size, dev)
    tables = maps.BlockTables(B, -(-longest // block_size), blocks, block_size, dev)
    follows = list(range(V))                                                             # the drafter
    ended = torch.zeros(B, dtype=torch.uint8, device=dev)
    no_drafts = torch.empty((B, 0), dtype=torch.int32, device=dev)

    def step(tokens, grow, total, max_q, done=None):
        """Feeds `total` tokens, grow[b] of them to request b; the attention's output, and what the tables gave."""
        s = tables.step(grow, total, done)
        maps.kv_append(cache, model.k[tokens], model.v[tokens], s.slots, tables.dev_err)
        out, _ = maps.kv_attend(cache, model.q[tokens], tables.table, tables.lens, s.tok_off, max_q, model.scale,
                                dev_err=tables.dev_err, granted=s.granted)
        return out, s

    def verify(target, drafted, n_draft):
        u = torch.rand(drafted.shape, generator=g, device=dev)
        noise = torch.empty((B, V), device=dev).exponential_(generator=g)
        return maps.verify_drafts(target, drafted, n_draft, u, noise, dev_err=tables.dev_err)

    # prompts: the last token of each gives the first answer's distribution
    lens = torch.tensor([len(p) for p in prompts], dtype=torch.int32, device=dev)
    flat = torch.tensor([x for p in prompts for x in p], device=dev)
    out, s = step(flat, lens, flat.numel(), max(map(len, prompts)))
    target = model.probabilities(out[s.tok_off[1:] - 1])[:, None]
    first, _ = verify(target, no_drafts, torch.zeros(B, dtype=torch.int32, device=dev))
    answers = first.tolist()                                                             # [B][1]

    steps = 1
    live = [new_tokens > 1] * B
    while any(live):
        alive = torch.tensor(live, device=dev)
        rows = alive.nonzero().squeeze(1)
        chain = [[a[-1]] for a in answers]                                               # the last token and the drafts
        for c in chain:
            for _ in range(K):
                c.append(follows[c[-1]])
        chain = torch.tensor(chain, dtype=torch.int32, device=dev)                       # [B, K + 1]
        fed = chain[rows].flatten().long()
        grow = torch.where(alive, K + 1, 0).to(torch.int32)
        done = (~alive).to(torch.uint8) & (1 - ended)                                    # give their blocks back, once
        ended |= done
        out, s = step(fed, grow, fed.numel(), K + 1, done)
        target = torch.zeros((B, K + 1, V), device=dev)
        target[rows] = model.probabilities(out).unflatten(0, (-1, K + 1))
        fed_to = alive & (s.granted != 0)     # (a refused request tries again; this cache has room for all)
        n_draft = torch.where(fed_to, K, -1).to(torch.int32)
        tokens, accepted = verify(target, chain[:, 1:].contiguous(), n_draft)
        # the rejected drafts' places are used again
        tables.lens -= torch.where(fed_to, K - accepted, 0).to(torch.int32)
        steps += 1
        for b, (n, row) in enumerate(zip(accepted.tolist(), tokens.tolist())):
            if n < 0:
                continue
            for x, y in zip(answers[b][-1:] + row[:n], row[:n + 1]):
                follows[x] = y
            answers[b] += row[:n + 1]
            live[b] = len(answers[b]) < new_tokens
    maps.check_errors(tables.dev_err)
    return [a[:new_tokens] for a in answers], steps


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    p.add_argument("--drafts", type=int, default=3)
    p.add_argument("--new-tokens", type=int, default=64)
    a = p.parse_args()
    g = torch.Generator().manual_seed(1)
    prompts = [torch.randint(0, 500, (n,), generator=g).tolist() for n in (5, 300, 41, 1, 128)]
    answers, steps = serve(Model.random(temperature=0.5), prompts, a.new_tokens, a.drafts, 1 << 20)
    for prompt, answer in zip(prompts, answers):
        print(f"{len(prompt)} prompt tokens -> {answer}")
    print(f"{len(prompts)} x {a.new_tokens} tokens in {steps} steps")


if __name__ == "__main__":
    main()
