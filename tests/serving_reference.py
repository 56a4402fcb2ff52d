"""Plain forms of the 4-bit cache and of verification, in 64 bits and on the CPU,
for the tests."""
from __future__ import annotations

import math

import torch

LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def quantise(x):
    """[..., D] values -> codes [..., D] (0 .. 15), scale bytes [..., D / 32], by the
    definition: the least scale 2^k with |x| <= 7 scale, k in -126 .. 125; the
    nearest level of x / scale, ties to the even code."""
    g = x.double().unflatten(-1, (-1, 32))
    finite = torch.isfinite(g).all(-1)
    top = torch.where(finite, g.abs().amax(-1), 0.0)
    k = torch.full(top.shape, -126, dtype=torch.int64)
    for e in range(-126, 125):
        k = torch.where(top > 7.0 * 2.0 ** e, e + 1, k)
    byte = torch.where(finite, k + 127, 255)
    y = torch.where(finite[..., None], g, 0.0) / (2.0 ** k.double())[..., None]
    a = y.abs()
    code = torch.zeros(a.shape, dtype=torch.int64)
    for i in range(1, 8):
        border = (LEVELS[i - 1] + LEVELS[i]) / 2
        code = torch.where((a > border) | ((a == border) & (i % 2 == 0)), i, code)
    code = code + 8 * torch.signbit(y)
    return code.flatten(-2), byte


def dequantise(code, byte):
    """The values, float64; NaN where the scale byte says so."""
    value = torch.tensor(LEVELS + [-v for v in LEVELS], dtype=torch.float64)[code.long()]
    unit = torch.where(byte.long() > 252, math.nan, 2.0 ** (byte.double() - 127.0))
    return (value.unflatten(-1, (-1, 32)) * unit[..., None]).flatten(-2)


def pack(code):
    return (code[..., 0::2] | code[..., 1::2] << 4).to(torch.uint8)


def unpack(b):
    b = b.long()
    return torch.stack([b & 15, b >> 4], -1).flatten(-2)


def row(logits, temperature):
    """A row's probabilities, or None where it is no distribution."""
    z = logits.double()
    if torch.isnan(z).any() or z.max() == math.inf or z.max() == -math.inf:
        return None
    t = float(torch.tensor(temperature, dtype=torch.float32))
    if not t >= 2.0 ** -60:
        p = torch.zeros_like(z)
        p[int(torch.nonzero(z == z.max())[0])] = 1.0
        return p
    w = torch.exp((z - z.max()) / min(t, 2.0 ** 60))
    return w / w.sum()


def verify(tokens, parents, logits, draft, temperature, uniforms, sample, distinct=False, most=None):
    """One request: (path, next token).  logits, draft: [tokens][vocab]."""
    n, vocab = len(tokens), logits.shape[1]
    if n == 0:
        return [], -1
    greedy = not temperature >= 2.0 ** -60
    path = [0]
    while True:
        node = path[-1]
        p = row(logits[node], temperature)
        if p is None:
            return path, -1
        whole, found = p.clone(), None
        kids = [i for i in range(node + 1, n) if (i - 1 if parents is None else parents[i]) == node]
        if most is not None and len(path) == most:
            kids = []
        q = None
        if draft is not None and not greedy and kids:
            q = row(draft[node], temperature)
            if q is None:
                kids = []
        for i in kids:
            x = tokens[i]
            known = 0 <= x < vocab
            if q is None:
                if known and float(uniforms[i]) * float(p.sum()) < float(p[x]):
                    found = i
                    break
                if known:
                    p[x] = 0.0
                continue
            if known and float(uniforms[i]) * float(q[x]) < float(p[x]):
                found = i
                break
            p = torch.clamp(p - q, min=0.0)
            if float(p.sum()) > 0.0:
                p = p / p.sum()
            if distinct and known:
                gone = float(q[x])
                q[x] = 0.0
                if gone < 1.0:
                    q = q / (1.0 - gone)
        if found is None:
            break
        path.append(found)
    if float(p.sum()) <= 0.0:
        p = whole
    upto = torch.cumsum(p, 0)
    return path, int(torch.searchsorted(upto, torch.tensor(float(sample), dtype=torch.float64) * upto[-1],
                                        right=True))
