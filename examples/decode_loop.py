"""A decode engine's loop over the paged cache, with every operator where it is used:

    kvx_repack      the prompts' KV arrive in the engine's pages
    kvx_append      per step and layer: the drafted tokens' queries and keys are
                    turned, their keys and values written behind the context
    kvx_attend      the drafted tree attends to its request's slots and its own branch
    kvx_commit      what verification accepted moves to the front of the draft
    kvx_weigh       the accepted tokens' attention weights add up per slot
    kvx_evict       a request over its budget keeps the slots of the largest weights

The model is a stand-in (random projections, a random accepted path): what it shows
is the order of the calls, the shapes, and what lives on the device.

    python examples/decode_loop.py
"""
from __future__ import annotations

import os
import random
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2509_17542_amd as K  # noqa: E402

LAYERS, HEADS, GROUP, DIM, PAGE = 2, 2, 2, 64, 16
Q_HEADS = HEADS * GROUP
BUDGET, SINK, RECENT = 96, 4, 32


def int32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Engine:
    """Requests that share one pool; every request owns `pages` pages."""

    def __init__(self, prompts, pages, seed=0):
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.rnd = random.Random(seed)
        self.requests = len(prompts)
        blocks = self.requests * pages + 1
        order = torch.randperm(blocks, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
        self.table = order[:self.requests * pages].view(self.requests, pages).cuda()
        self.cache = torch.zeros((LAYERS, 2, blocks, PAGE, HEADS, DIM), dtype=torch.bfloat16, device="cuda")
        # prefill's buffers, token-major, requests back to back
        shard = torch.randn(2 * LAYERS * sum(prompts) * HEADS * DIM, generator=self.gen, device="cuda").bfloat16()
        plan = K.kvx_plan(K.make_desc(LAYERS, HEADS, DIM, 1, 1, 0, K.BF16, K.BF16, K.THD, PAGE, blocks, prompts))
        K.kvx_repack(plan, [shard], self.cache, None, self.table, pages)
        self.view = K.make_cache(self.cache, None, self.table)
        self.slots = pages * PAGE
        self.lens = list(prompts)              # slots in use
        self.placed = list(prompts)            # positions given out: eviction does not take them back
        self.weights = torch.zeros((LAYERS, self.requests, HEADS, self.slots), device="cuda")
        self.inv_freq = 10000.0 ** (-torch.arange(0, DIM, 2, device="cuda", dtype=torch.float32) / DIM)
        self.scores = K.make_scores(DIM ** -0.5)

    def normal(self, *shape):
        return torch.randn(shape, generator=self.gen, device="cuda")

    def draft(self, nodes):
        """A random tree of `nodes` tokens for every request: parents, and each
        token's ancestors as bits."""
        parents, bits, depth = [], [], []
        for _ in range(self.requests):
            tree, rows, deep = [], [], []
            for i in range(nodes):
                p = self.rnd.randint(max(-1, i - 3), i - 1)
                tree.append(p)
                rows.append((rows[p] if p >= 0 else 0) | 1 << i)
                deep.append(deep[p] + 1 if p >= 0 else 0)
            parents.append(tree)
            bits += rows
            depth += deep
        return parents, torch.tensor(bits, dtype=torch.int64, device="cuda")[:, None], depth

    def step(self, nodes):
        parents, tree, depth = self.draft(nodes)
        n = self.requests * nodes
        starts = int32([nodes * r for r in range(self.requests + 1)])
        contexts = int32(self.lens)
        place = [self.placed[i // nodes] + d for i, d in enumerate(depth)]
        longest = max(self.lens) + nodes
        batch = K.make_batch(starts, contexts, n, nodes, longest, tree=tree)
        rope = K.make_rope(self.inv_freq, [DIM // 2], int32([place]))
        workspace = torch.empty(max(16, K.kvx_attend_workspace(self.view, batch, Q_HEADS)), dtype=torch.uint8,
                                device="cuda")
        turned, lse, out = [], [], None
        for layer in range(LAYERS):
            qkv = self.normal(n, Q_HEADS + 2 * HEADS, DIM).bfloat16()
            q, k, v = qkv.split([Q_HEADS, HEADS, HEADS], dim=1)
            out = torch.empty((n, Q_HEADS, DIM), dtype=torch.bfloat16, device="cuda")
            z = torch.empty((n, Q_HEADS), device="cuda")
            K.kvx_append(self.view, batch, rope, layer, q, k, v, q)
            K.kvx_attend(self.view, batch, self.scores, layer, q, out, z, workspace)
            turned.append(q)
            lse.append(z)
        # verification: the path to a random node is accepted
        paths = []
        for tree_of in parents:
            node, path = self.rnd.randrange(nodes), []
            while node >= 0:
                path.append(node)
                node = tree_of[node]
            paths.append(path[::-1])
        most = max(map(len, paths))
        accepted = int32([p + [0] * (most - len(p)) for p in paths])
        counts = int32([len(p) for p in paths])
        new_lens = torch.empty_like(contexts)
        K.kvx_commit(self.view, 0, LAYERS, contexts, accepted, counts, new_lens)
        # an accepted token saw the context and its own path: the slots it now lies behind
        rows = torch.tensor([r * nodes + i for r, p in enumerate(paths) for i in p], device="cuda")
        ends = [0]
        for p in paths:
            ends.append(ends[-1] + len(p))
        chain = K.make_batch(int32(ends), contexts, ends[-1], most, longest)
        for layer in range(LAYERS):
            K.kvx_weigh(self.view, chain, self.scores, layer, turned[layer][rows].contiguous(),
                        lse[layer][rows].contiguous(), self.weights[layer])
        self.lens = [c + len(p) for c, p in zip(self.lens, paths)]
        self.placed = [c + len(p) for c, p in zip(self.placed, paths)]
        assert new_lens.tolist() == self.lens
        return out

    def evict(self):
        """Requests over the budget keep BUDGET slots of every layer and head.  The kept
        keys stay turned by their old positions; a window or a bias (this engine has
        none) would go by slots from here on."""
        kept = torch.empty((LAYERS, self.requests, HEADS, BUDGET), dtype=torch.int32, device="cuda")
        new_lens = torch.empty(self.requests, dtype=torch.int32, device="cuda")
        K.kvx_evict(self.view, 0, LAYERS, int32(self.lens), max(self.lens), BUDGET, SINK, RECENT, self.weights,
                    self.weights, kept, new_lens)
        self.lens = new_lens.tolist()
        return kept


def main(steps=20, nodes=8):
    engine = Engine([40, 57, 90], pages=10)
    for step in range(steps):
        out = engine.step(nodes)
        line = f"step {step:2d}: slots in use {engine.lens}"
        if max(engine.lens) > BUDGET + PAGE:
            engine.evict()
            line += f", after eviction {engine.lens}"
        print(line)
    torch.cuda.synchronize()
    assert torch.isfinite(out.float()).all()
    return engine


if __name__ == "__main__":
    main()
