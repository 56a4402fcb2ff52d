"""A decode engine's loop over the paged cache, with every operator where it is used:

    kvx_repack      the prompts' KV arrive in the engine's pages (a cache of 4 bits takes them
                    by kvx_append, as they are quantised)
    kvx_append      per step and layer: the drafted tokens' queries and keys are
                    turned, their keys and values written behind the context
    kvx_attend      the drafted tree attends to its request's slots and its own branch
    kvx_verify      the drafted tokens against the target's logits: the accepted path and the
                    token that follows it, which the next tree starts from
    kvx_commit      the path moves to the front of the draft
    kvx_weigh       the accepted tokens' attention weights add up per slot
    kvx_evict       a request over its budget keeps the slots of the largest weights
    kvx_fetch       a conversation's rows read back into 16 bits, as another instance wants them

The model is a stand-in (random projections and logits): what it shows is the order of
the calls, the shapes, and what lives on the device.  Over a cache of 4 bits slots are
not weighed, and none are evicted.

    python examples/decode_loop.py [--four]
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
VOCAB, TEMPERATURE = 1000, 0.8


def int32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Engine:
    """Requests that share one pool; every request owns `pages` pages."""

    def __init__(self, prompts, pages, seed=0, four=False):
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.rnd = random.Random(seed)
        self.requests = len(prompts)
        blocks = self.requests * pages + 1
        order = torch.randperm(blocks, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
        self.table = order[:self.requests * pages].view(self.requests, pages).cuda()
        # prefill's buffers, token-major, requests back to back
        total = sum(prompts)
        shard = torch.randn(2 * LAYERS * total * HEADS * DIM, generator=self.gen, device="cuda").bfloat16()
        self.four = four
        if four:
            shape = (LAYERS, 2, blocks, PAGE, HEADS)
            self.cache = torch.zeros((*shape, DIM // 2), dtype=torch.uint8, device="cuda")
            self.scale_bytes = torch.full((*shape, DIM // 32), 127, dtype=torch.uint8, device="cuda")
            self.view = K.make_cache(self.cache, self.scale_bytes, self.table, dtype=K.E2M1)
            starts = [sum(prompts[:r]) for r in range(self.requests + 1)]
            batch = K.make_batch(int32(starts), int32([0] * self.requests), total, max(prompts), max(prompts))
            turned = K.make_rope(torch.zeros(0, device="cuda"), [0], torch.zeros((1, total), dtype=torch.int32, device="cuda"))
            at = 0
            rows = torch.empty((LAYERS, 2, total, HEADS, DIM), dtype=torch.bfloat16, device="cuda")
            for r, n in enumerate(prompts):
                size = 2 * LAYERS * n * HEADS * DIM
                rows[:, :, starts[r]:starts[r + 1]] = shard[at:at + size].view(LAYERS, 2, n, HEADS, DIM)
                at += size
            for layer in range(LAYERS):
                K.kvx_append(self.view, batch, turned, layer, None, rows[layer, 0], rows[layer, 1], None)
        else:
            self.cache = torch.zeros((LAYERS, 2, blocks, PAGE, HEADS, DIM), dtype=torch.bfloat16, device="cuda")
            plan = K.kvx_plan(K.make_desc(LAYERS, HEADS, DIM, 1, 1, 0, K.BF16, K.BF16, K.THD, PAGE, blocks, prompts))
            K.kvx_repack(plan, [shard], self.cache, None, self.table, pages)
            self.view = K.make_cache(self.cache, None, self.table)
        self.last = [self.rnd.randrange(VOCAB) for _ in prompts]       # sampled, not in the cache yet
        self.slots = pages * PAGE
        self.lens = list(prompts)              # slots in use
        self.placed = list(prompts)            # positions given out: eviction does not take them back
        self.weights = torch.zeros((LAYERS, self.requests, HEADS, self.slots), device="cuda")
        self.inv_freq = 10000.0 ** (-torch.arange(0, DIM, 2, device="cuda", dtype=torch.float32) / DIM)
        self.scores = K.make_scores(DIM ** -0.5)

    def normal(self, *shape):
        return torch.randn(shape, generator=self.gen, device="cuda")

    def draft(self, nodes):
        """A random tree of `nodes` tokens for every request, the first of them the one
        sampled last: parents, and each token's ancestors as bits."""
        parents, bits, depth = [], [], []
        for _ in range(self.requests):
            tree, rows, deep = [], [], []
            for i in range(nodes):
                p = self.rnd.randint(max(0, i - 3), i - 1) if i else -1
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
        # the model's head, and what a small model drafted: mostly tokens that the target likes
        logits = 2.0 * self.normal(n, VOCAB)
        tokens = [self.rnd.randrange(VOCAB) for _ in range(n)]
        for r, tree_of in enumerate(parents):
            tokens[r * nodes] = self.last[r]
            for i in range(1, nodes):
                logits[r * nodes + tree_of[i], tokens[r * nodes + i]] += 6.0
        drafts = K.make_drafts(starts, int32(tokens), nodes, VOCAB, parents=int32(sum(parents, [])),
                               temperatures=torch.full((self.requests,), TEMPERATURE, device="cuda"))
        accepted = torch.empty((self.requests, nodes), dtype=torch.int32, device="cuda")
        counts, following = (torch.empty_like(contexts) for _ in range(2))
        space = torch.empty(max(16, K.kvx_verify_workspace(drafts, False)), dtype=torch.uint8, device="cuda")
        K.kvx_verify(drafts, logits.bfloat16(), None, torch.rand(n, generator=self.gen, device="cuda"),
                     torch.rand(self.requests, generator=self.gen, device="cuda"), accepted, counts, following, space)
        new_lens = torch.empty_like(contexts)
        K.kvx_commit(self.view, 0, LAYERS, contexts, accepted, counts, new_lens)
        paths = [path[:c] for path, c in zip(accepted.tolist(), counts.tolist())]
        most = max(map(len, paths))
        self.last = following.tolist()
        # an accepted token saw the context and its own path: the slots it now lies behind
        rows = torch.tensor([r * nodes + i for r, p in enumerate(paths) for i in p], device="cuda")
        ends = [0]
        for p in paths:
            ends.append(ends[-1] + len(p))
        chain = K.make_batch(int32(ends), contexts, ends[-1], most, longest)
        for layer in range(0 if self.four else LAYERS):
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

    def rows(self, r, layer):
        """The keys and values of a request's slots, [slots][heads][dim] in bfloat16."""
        lens = [n if i == r else 0 for i, n in enumerate(self.lens)]
        starts = [sum(lens[:i]) for i in range(self.requests + 1)]
        batch = K.make_batch(int32(starts), int32([0] * self.requests), lens[r], lens[r], lens[r])
        k, v = (torch.empty((lens[r], HEADS, DIM), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        K.kvx_fetch(self.view, batch, layer, k, v)
        return k, v


def main(steps=20, nodes=8, four=False):
    engine = Engine([40, 57, 90], pages=24 if four else 10, four=four)
    for step in range(steps):
        out = engine.step(nodes)
        line = f"step {step:2d}: slots in use {engine.lens}"
        if not four and max(engine.lens) > BUDGET + PAGE:
            engine.evict()
            line += f", after eviction {engine.lens}"
        print(line)
    torch.cuda.synchronize()
    assert torch.isfinite(out.float()).all()
    return engine


if __name__ == "__main__":
    main(four="--four" in sys.argv[1:])
