"""Plain 64-bit forms of the decode operators and the problems that their tests
run: small caches with every unused slot and page poisoned, so that a read
outside a request's slots shows."""
from __future__ import annotations

import math
import random

import torch

FLOAT8 = {"e4m3fn": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
TORCH = {"fp16": torch.float16, "bf16": torch.bfloat16, **FLOAT8}
FMAX = {"e4m3fn": 448.0, "e5m2": 57344.0}
UNIT = {"fp16": 2.0 ** -11, "bf16": 2.0 ** -8}      # unit roundoff


class Problem:
    """One cache and one batch.  `new` and `ctx`: new tokens and slots in use of
    each request; `tree`: None, or a seed of random trees; `values` scales q and k."""

    def __init__(self, new, ctx, heads=2, group=2, dim=64, dtype="bf16", cache="bf16", page=16,
                 layers=1, layer=0, tree=None, softcap=0.0, slopes=False, window=0, prefix=None,
                 seed=0, values=1.0, blocks=None, positions=None, poison=math.nan, spare=0):
        self.__dict__.update(new=list(new), ctx=list(ctx), heads=heads, group=group, dim=dim,
                             dtype=dtype, kind=cache, page=page, layers=layers, layer=layer,
                             softcap=softcap, window=window, prefix=prefix, q_heads=heads * group)
        g = torch.Generator().manual_seed(seed)
        self.total = [a + b for a, b in zip(new, ctx)]
        R = len(new)
        self.max_context = max(max(self.total, default=1), 1)
        self.max_tokens = max(max(new, default=1), 1)
        pages = [-(-(t + spare) // page) for t in self.total]
        need = sum(pages)
        self.blocks = blocks or need + 2
        order = torch.randperm(self.blocks, generator=g)[:need].tolist()
        self.stride = max(max(pages, default=1), 1)
        self.table = torch.full((R, self.stride), -1, dtype=torch.int32)
        for r, n in enumerate(pages):
            for k in range(n):
                self.table[r, k] = order.pop()
        shape = (layers, 2, self.blocks, page, heads, dim)
        x = torch.randn(shape, generator=g) * (0.25 + torch.rand((1, 2, 1, 1, heads, 1), generator=g))
        x[:, 0] *= values
        used = torch.zeros(self.blocks, page, dtype=torch.bool)
        for r, t in enumerate(self.total):
            for j in range(t):
                used[self.table[r, j // page], j % page] = True
        if cache in FLOAT8:
            s = x.abs().amax(-1) / FMAX[cache]
            code = (x / s[..., None]).to(FLOAT8[cache])
            s[:, :, ~used] = poison
            bits = code.view(torch.uint8)
            bits[:, :, ~used] = 0x7F
            self.cache, self.scales = bits.view(FLOAT8[cache]), s
        else:
            x[:, :, ~used] = poison
            self.cache, self.scales = x.to(TORCH[cache]), None
        N = sum(new)
        self.tokens = N
        self.starts = [sum(new[:r]) for r in range(R + 1)]
        self.q = (torch.randn((N, self.q_heads, dim), generator=g) * values).to(TORCH[dtype])
        self.scale = 1.0 / math.sqrt(dim)
        self.slopes = (0.02 + torch.rand(self.q_heads, generator=g)) if slopes else None
        self.tree = self.positions = None
        if tree is not None:
            rnd = random.Random(tree)
            words = (self.max_tokens + 63) // 64
            self.tree = torch.zeros((N, words), dtype=torch.int64)
            pos = []
            for r, n in enumerate(new):
                sets = []
                for i in range(n):
                    p = rnd.randint(max(-1, i - 6), i - 1)
                    sets.append((sets[p] if p >= 0 else set()) | {i})
                    pos.append(ctx[r] + len(sets[i]) - 1)
                    for j in sets[i]:
                        bit = 1 << j % 64
                        self.tree[self.starts[r] + i, j // 64] |= bit - (1 << 64 if bit >> 63 else 0)
            self.positions = torch.tensor(pos, dtype=torch.int32)
        if positions is not None:
            self.positions = torch.tensor(positions, dtype=torch.int32)

    # -- what a request holds --

    def slot(self, r, j):
        return int(self.table[r, j // self.page]), j % self.page

    def rows(self, kv, r):
        """[slots][heads][dim] of request r as 64-bit values."""
        at = torch.arange(self.total[r])
        page = self.table[r].long()[at // self.page] if self.total[r] else at
        ok = (page >= 0) & (page < self.blocks)
        page = torch.where(ok, page, 0)
        bits = self.cache.view(torch.uint8 if self.scales is not None else torch.int16)
        x = bits[self.layer, kv][page, at % self.page].view(self.cache.dtype).double()
        if self.scales is not None:
            x = x * self.scales[self.layer, kv][page, at % self.page].double()[..., None]
        return x, ok

    def place(self, r, j):
        """Position of slot j of request r."""
        if j >= self.ctx[r] and self.positions is not None:
            return int(self.positions[self.starts[r] + j - self.ctx[r]])
        return j

    def sees(self, r, i):
        """Which slots token i of request r sees, and its distance to each."""
        T, C = self.total[r], self.ctx[r]
        tok = self.starts[r] + i
        at = torch.arange(T)
        mine = int(self.positions[tok]) if self.positions is not None else C + i
        pos = at.clone()
        if self.positions is not None:
            pos[C:] = self.positions[self.starts[r]:self.starts[r] + T - C].long()
        see = at <= C + i
        if self.tree is not None:
            see = at < C
            for j in range(T - C):
                see[C + j] = bool(int(self.tree[tok, j // 64]) >> (j % 64) & 1)
        distance = mine - pos
        if self.window:
            see &= distance < self.window
        if self.prefix is not None:
            see |= at < int(self.prefix[r])
        return see, distance

    def gpu(self, K):
        """(view, batch, scores) on the device."""
        dev = lambda x: None if x is None else x.cuda()  # noqa: E731
        self.d_cache, self.d_scales = dev(self.cache), dev(self.scales)
        view = K.make_cache(self.d_cache, self.d_scales, self.table.cuda())
        batch = K.make_batch(torch.tensor(self.starts, dtype=torch.int32).cuda(),
                             torch.tensor(self.ctx, dtype=torch.int32).cuda(), self.tokens,
                             self.max_tokens, self.max_context, positions=dev(self.positions),
                             tree=dev(self.tree))
        prefix = None if self.prefix is None else torch.tensor(self.prefix, dtype=torch.int32).cuda()
        return view, batch, K.make_scores(self.scale, softcap=self.softcap, slopes=dev(self.slopes),
                                          window=self.window, prefix=prefix)


def attend(p):
    """out, lse in 64 bits; and for each row the sum of |p v| and a bound of its
    scores' error, which the tolerances are derived from."""
    shape = (p.tokens, p.q_heads)
    out = torch.zeros((*shape, p.dim), dtype=torch.float64)
    size = torch.zeros((*shape, p.dim), dtype=torch.float64)
    lse = torch.full(shape, -math.inf, dtype=torch.float64)
    delta = torch.zeros(shape, dtype=torch.float64)
    q = p.q.double()
    for r, n in enumerate(p.new):
        k, ok = p.rows(0, r)
        v, _ = p.rows(1, r)
        for i in range(n):
            tok = p.starts[r] + i
            see, distance = p.sees(r, i)
            idx = torch.nonzero(see & ok)[:, 0]
            if not len(idx):
                continue
            qi = q[tok].view(p.heads, p.group, p.dim)
            kk, vv = k[idx].permute(1, 2, 0), v[idx].permute(1, 0, 2)
            x = torch.matmul(qi, kk) * p.scale
            # products are exact in fp32 or rounded once, D of them summed
            d = (torch.matmul(qi.abs(), kk.abs()) * p.scale).amax(-1) * (p.dim + 8) * 2.0 ** -24
            if p.softcap:
                x = p.softcap * torch.tanh(x / p.softcap)
            if p.slopes is not None:
                x = x - p.slopes.double().view(p.heads, p.group, 1) * distance[idx].abs().double()
            d = d + x.abs().amax(-1) * 2.0 ** -21 + p.softcap * 2.0 ** -21
            z = torch.logsumexp(x, -1)
            w = torch.exp(x - z[..., None])
            out[tok] = torch.matmul(w, vv).reshape(p.q_heads, p.dim)
            size[tok] = torch.matmul(w, vv.abs()).reshape(p.q_heads, p.dim)
            lse[tok], delta[tok] = z.reshape(-1), d.reshape(-1)
    return out, lse, size, delta


def weigh(p, lse, start):
    """The accumulated weights, and a bound of their error."""
    w = start.double().clone()
    err = torch.zeros_like(w)
    q = p.q.double()
    for r, n in enumerate(p.new):
        C, T = p.ctx[r], p.total[r]
        w[r, :, C:T] = 0
        k, ok = p.rows(0, r)
        k = torch.where(ok[:, None, None], k, 0.0)
        for i in range(n):
            tok = p.starts[r] + i
            see, distance = p.sees(r, i)
            idx = torch.nonzero(see & ok)[:, 0]
            if not len(idx):
                continue
            qi = q[tok].view(p.heads, p.group, p.dim)
            kk = k[idx].permute(1, 2, 0)
            x = torch.matmul(qi, kk) * p.scale
            d = torch.matmul(qi.abs(), kk.abs()) * p.scale * (p.dim + 8) * 2.0 ** -24
            if p.softcap:
                x = p.softcap * torch.tanh(x / p.softcap)
            if p.slopes is not None:
                x = x - p.slopes.double().view(p.heads, p.group, 1) * distance[idx].abs().double()
            l64 = lse[tok].double().view(p.heads, p.group, 1)
            d = d + x.abs() * 2.0 ** -21 + l64.abs() * 2.0 ** -23 + p.softcap * 2.0 ** -21 + 2.0 ** -21
            e = torch.where(l64 == -math.inf, 0.0, torch.exp(x - l64))
            w[r][:, idx] += e.sum(1)
            err[r][:, idx] += torch.where(e == 0.0, 0.0, 2 * d * e).sum(1)
    # fp32 sums of at most tokens x group terms and the old weight
    return w, err + w.abs() * 2.0 ** -20 + 1e-30


def evict(T, budget, sink, recent, w):
    """The slots that stay, ascending, of one (layer, request, head)."""
    if T <= budget:
        return list(range(T))
    key = [(math.inf, 1) if math.isnan(float(x)) else (float(x), 0) for x in w[:T]]
    rest = sorted(range(sink, T - recent), key=lambda j: (-key[j][0], -key[j][1], j))
    stay = list(range(sink)) + list(range(T - recent, T)) + rest[:budget - sink - recent]
    return sorted(stay)


def rotate(x, inv_freq, sections, positions, interleaved):
    """x [tokens][heads][dim] turned, in 64 bits from the fp32 angles."""
    x = x.double().clone()
    pairs = len(inv_freq)
    axis = [a for a, n in enumerate(sections) for _ in range(n)]
    angle = (positions.float()[axis].T * inv_freq[None, :]).double() if pairs else \
        torch.zeros((x.shape[0], 0), dtype=torch.float64)
    c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    if interleaved:
        ia, ib = slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)
    else:
        ia, ib = slice(0, pairs), slice(pairs, 2 * pairs)
    a, b = x[..., ia].clone(), x[..., ib].clone()
    x[..., ia], x[..., ib] = a * c - b * s, b * c + a * s
    return x
