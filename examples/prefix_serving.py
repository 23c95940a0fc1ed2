#!/usr/bin/env python3
"""Serving with a prefix cache in device memory: the index and the paged-cache operators together.

A server keeps the keys and values of 16-token blocks in one pool, [block, layer, keys or values, token, KV head, element], and an LSM index
that maps the key of a block (a digest of all tokens up to its end) to the block's number.  For a batch of requests it

  1. looks all their block keys up (LsmDriver.probe): the longest cached prefix of each request, as block numbers;
  2. groups requests whose cached prefixes begin alike: what they share is read once for all of them;
  3. runs the layers over the tokens that are not cached: lsm_kv_append norms and rotates queries and keys and puts keys and values
     into the pool, lsm_prefix_attention attends over the shared prefix and each request's own blocks;
  4. enters the new complete blocks into the index (LsmDriver.flush_unsorted), where later batches find them;
  5. decodes: one token per request and step, over the same pages.

The model is a stack of attention layers with random weights; nothing is learned or loaded.

  python examples/prefix_serving.py            (on an MI355X)
"""
from __future__ import annotations

import os
import sys
import time
from dataclasses import dataclass, field
from typing import List

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2511_16138_amd as lsm  # noqa: E402
from workloads import keys as K  # noqa: E402

BLOCK = 16  # tokens


@dataclass
class Request:
    tokens: List[int]
    blocks: List[int] = field(default_factory=list)  # pool blocks of its tokens
    cached: int = 0                                  # tokens whose keys and values are in the pool
    found: int = 0                                   # of these, how many the index had


class Server:
    def __init__(self, layers=4, heads=32, kv_heads=2, head_dim=128, width=1024, vocab=1000, blocks=4096, max_tokens=4096, dtype=torch.bfloat16, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *shape: torch.randn(shape, generator=gen, device="cuda")  # noqa: E731
        self.layers, self.heads, self.kv_heads, self.head_dim = layers, heads, kv_heads, head_dim
        self.embedding = rand(vocab, width).to(dtype)
        self.qkv = [(rand(width, (heads + 2 * kv_heads) * head_dim) / width ** 0.5).to(dtype) for _ in range(layers)]
        self.out = [(rand(heads * head_dim, width) / (heads * head_dim) ** 0.5).to(dtype) for _ in range(layers)]
        self.q_norm, self.k_norm = ([(1 + 0.1 * rand(head_dim)).to(dtype) for _ in range(layers)] for _ in range(2))
        self.table = lsm.lsm_rope_table(max_tokens, head_dim)
        self.pool = torch.zeros((blocks, layers, 2, BLOCK, kv_heads, head_dim), dtype=dtype, device="cuda")
        self.free = list(range(blocks))
        self.index = lsm.LsmDriver(buffer_entries=1024, bloom_bits=16)
        self.seqno = 0

    # -- index ----------------------------------------------------------------------------------------------------
    @staticmethod
    def block_keys(requests: List[Request]):
        """Keys of the complete blocks of every request: int64 [requests, blocks, 4] as the index stores them, and their counts."""
        counts = [min(len(r.tokens) // BLOCK, lsm.binding.LSM_MAX_BLOCKS) for r in requests]
        most = max(counts + [1])
        tokens = torch.zeros((len(requests), most, BLOCK), dtype=torch.int64)
        for i, (r, c) in enumerate(zip(requests, counts)):
            tokens[i, :c] = torch.tensor(r.tokens[:c * BLOCK], dtype=torch.int64).reshape(c, BLOCK)
        words = K.key_bytes_words(K.chain_keys(tokens).reshape(-1, 4)).reshape(len(requests), most, 4)
        return words.cuda(), torch.tensor(counts, dtype=torch.int32, device="cuda")

    def look_up(self, requests: List[Request]) -> None:
        keys, counts = self.block_keys(requests)
        hit_len, hits = self.index.probe(keys, counts)
        blocks = (hits[..., 0] & 0xFFFFFFFF).tolist()  # value pointer = block number
        for r, n, found in zip(requests, hit_len.tolist(), blocks):
            n = max(0, min(n, (len(r.tokens) - 1) // BLOCK))  # at least one token has to be run for its output
            r.blocks, r.cached, r.found = found[:n], n * BLOCK, n * BLOCK

    def enter(self, requests: List[Request]) -> None:
        """The complete blocks that the index did not have, one put each."""
        keys, counts = self.block_keys(requests)
        rows = []
        for i, (r, n) in enumerate(zip(requests, counts.tolist())):
            for b in range(r.found // BLOCK, min(n, r.cached // BLOCK)):
                rows.append((i, b, r.blocks[b]))
        if rows:
            i, b, block = torch.tensor(rows, device="cuda").T
            entries = torch.zeros((len(rows), 8), dtype=torch.int64, device="cuda")
            entries[:, :4] = keys[i, b]
            entries[:, 4] = self.seqno + torch.arange(1, len(rows) + 1, device="cuda")
            entries[:, 6], entries[:, 7] = block, self.pool[0].numel() * self.pool.element_size()
            for part in entries.split(1024):
                self.index.flush_unsorted(part.contiguous())
            self.seqno += len(rows)

    # -- one pass over new tokens ---------------------------------------------------------------------------------
    def plan(self, requests: List[Request]):
        """The batch in an order in which requests that share blocks are neighbours: (order, PrefixBatch, positions, slots, new tokens)."""
        wanted = sum(max(0, -(-len(r.tokens) // BLOCK) - len(r.blocks)) for r in requests)
        if any(not 0 < len(r.tokens) <= self.table.shape[0] for r in requests) or wanted > len(self.free):
            raise ValueError(f"requests must have 1 to {self.table.shape[0]} tokens and fit the pool: {wanted} blocks wanted, {len(self.free)} free")
        for r in requests:
            while len(r.blocks) * BLOCK < len(r.tokens):
                r.blocks.append(self.free.pop())
        whole = [r.blocks[:r.cached // BLOCK] for r in requests]  # blocks that no new token is written to
        order = sorted(range(len(requests)), key=lambda i: whole[i])
        groups: List[List[int]] = []
        for i in order:
            if groups and whole[i] and whole[groups[-1][0]][:1] == whole[i][:1]:
                groups[-1].append(i)
            else:
                groups.append([i])
        prefix = []
        for g in groups:
            shared = whole[g[0]] if len(g) > 1 else []
            for i in g[1:]:
                n = 0
                while n < min(len(shared), len(whole[i])) and shared[n] == whole[i][n]:
                    n += 1
                shared = shared[:n]
            prefix.append(shared)
        ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731

        def table(rows):
            wide = max([len(r) for r in rows] + [0])
            return ints([r + [-1] * (wide - len(r)) for r in rows]).reshape(len(rows), wide)

        sums = lambda v: [sum(v[:i]) for i in range(len(v) + 1)]  # noqa: E731
        shares = [len(p) for p, g in zip(prefix, groups) for _ in g]
        new = [requests[i].tokens[requests[i].cached:] for i in order]
        batch = lsm.PrefixBatch(ints(sums([len(g) for g in groups])), table(prefix), ints([len(p) * BLOCK for p in prefix]), ints(sums([len(t) for t in new])),
                                table([requests[i].blocks[n:] for i, n in zip(order, shares)]),
                                ints([len(requests[i].tokens) - n * BLOCK for i, n in zip(order, shares)]))
        places = [(p, requests[i].blocks[p // BLOCK] * BLOCK + p % BLOCK) for i in order for p in range(requests[i].cached, len(requests[i].tokens))]
        positions, slots = torch.tensor(places, dtype=torch.int64, device="cuda").T.contiguous()
        return order, batch, positions.to(torch.int32), slots, torch.tensor([t for ts in new for t in ts], device="cuda")

    def forward(self, requests: List[Request]) -> torch.Tensor:
        """Runs every request's uncached tokens; the logits of each one's last token, float32 [requests, vocab]."""
        order, batch, positions, slots, tokens = self.plan(requests)
        x = self.embedding[tokens].float()
        h, kv = self.heads, self.kv_heads
        for l in range(self.layers):
            normed = (x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6)).to(self.embedding.dtype)
            fused = (normed @ self.qkv[l]).view(-1, h + 2 * kv, self.head_dim)
            k_pages, v_pages = self.pool[:, l, 0], self.pool[:, l, 1]
            q = lsm.lsm_kv_append(fused[:, h:h + kv], fused[:, h + kv:], positions, slots, k_pages, v_pages, self.table, k_weight=self.k_norm[l],
                                  q=fused[:, :h], q_weight=self.q_norm[l])
            o = lsm.lsm_prefix_attention(q, k_pages, v_pages, batch)
            x = x + (o.view(o.shape[0], -1) @ self.out[l]).float()
        last = x[batch.q_offsets[1:].long() - 1]
        for r in requests:
            r.cached = len(r.tokens)
        logits = torch.empty((len(requests), self.embedding.shape[0]), device="cuda")
        logits[torch.tensor(order, device="cuda")] = last @ self.embedding.float().T
        return logits

    def prefill(self, requests: List[Request]) -> torch.Tensor:
        self.look_up(requests)
        logits = self.forward(requests)
        self.enter(requests)
        return logits

    def decode(self, requests: List[Request], next_tokens: List[int]) -> torch.Tensor:
        for r, t in zip(requests, next_tokens):
            r.tokens.append(t)
        return self.forward(requests)


def main() -> None:
    server = Server()
    gen = torch.Generator().manual_seed(1)
    draw = lambda n: torch.randint(0, 1000, (n,), generator=gen).tolist()  # noqa: E731
    prompts = [draw(512), draw(1024)]
    for round_number in range(3):
        requests = [Request(prompts[i % 2] + draw(20 + 3 * i)) for i in range(16)]
        torch.cuda.synchronize()
        t = time.perf_counter()
        logits = server.prefill(requests)
        torch.cuda.synchronize()
        total, found = sum(len(r.tokens) for r in requests), sum(r.found for r in requests)
        print(f"batch {round_number}: {total} tokens, {found} of them found in the index, prefill {1e3 * (time.perf_counter() - t):.1f} ms")
        for _ in range(8):
            logits = server.decode(requests, logits.argmax(-1).tolist())
        print("  next tokens", logits.argmax(-1)[:8].tolist())


if __name__ == "__main__":
    main()
