"""The 4-bit cache: kvx_append quantises as the definition does, bit for bit, and
kvx_fetch reads back what is there, out of every type of cache; kvx_commit and
kvx_evict move its rows."""
import math

import pytest
import torch

import operator_reference as ops
import serving_reference as ref

pytestmark = pytest.mark.gpu
TORCH = {**ops.TORCH, "e2m1": torch.uint8}


@pytest.fixture(scope="module")
def K():
    import paper_2509_17542_amd as K
    return K


def int32(v):
    return torch.tensor(v, dtype=torch.int32).cuda()


class Pool:
    """A cache of `kind` full of poison, and a batch of `new` tokens behind `ctx`."""

    def __init__(self, K, new, ctx, heads=2, dim=64, kind="e2m1", page=16, layers=1, seed=0, fill=False):
        g = torch.Generator().manual_seed(seed)
        self.new, self.ctx, self.page, self.kind, self.dim = new, ctx, page, kind, dim
        pages = [max(1, -(-(a + b) // page)) for a, b in zip(new, ctx)]
        self.blocks = sum(pages) + 2
        order = torch.randperm(self.blocks, generator=g)[:sum(pages)].tolist()
        self.table = torch.full((len(new), max(pages)), -1, dtype=torch.int32)
        for r, n in enumerate(pages):
            for i in range(n):
                self.table[r, i] = order.pop()
        shape = (layers, 2, self.blocks, page, heads, dim)
        if kind == "e2m1":
            cache = torch.randint(0, 256, (*shape[:-1], dim // 2), generator=g, dtype=torch.uint8)
            scales = torch.randint(110, 140, (*shape[:-1], dim // 32), generator=g, dtype=torch.uint8)
        elif kind in ops.FLOAT8:
            cache = torch.randint(0, 256, shape, generator=g, dtype=torch.uint8).view(TORCH[kind])
            scales = torch.rand(shape[:-1], generator=g)
        else:
            cache, scales = torch.randn(shape, generator=g).to(TORCH[kind]), None
        self.cache, self.scales = cache.cuda(), None if scales is None else scales.cuda()
        self.before = self.cache.clone(), None if scales is None else self.scales.clone()
        self.view = K.make_cache(self.cache, self.scales, self.table.cuda(),
                                 dtype=K.E2M1 if kind == "e2m1" else None)
        self.tokens = sum(new)
        self.starts = [sum(new[:r]) for r in range(len(new) + 1)]
        total = [a + b for a, b in zip(new, ctx)]
        self.batch = K.make_batch(int32(self.starts), int32(ctx), self.tokens, max(max(new), 1), max(max(total), 1))

    def where(self):
        """(page, slot) of every token."""
        page, slot = [], []
        for r, n in enumerate(self.new):
            for i in range(n):
                j = self.ctx[r] + i
                page.append(int(self.table[r, j // self.page]))
                slot.append(j % self.page)
        return torch.tensor(page, dtype=torch.long), torch.tensor(slot, dtype=torch.long)


def no_rope(K, n):
    return K.make_rope(torch.zeros(0, device="cuda"), [0], torch.zeros((1, n), dtype=torch.int32, device="cuda"))


def append(K, p, k, v, layer=0):
    K.kvx_append(p.view, p.batch, no_rope(K, p.tokens), layer, None, k, v, None)


CASES = {
    "one": dict(new=[1], ctx=[0]),
    "tokens": dict(new=[1, 1, 1], ctx=[0, 15, 300]),
    "prompts": dict(new=[37, 0, 130], ctx=[0, 5, 64], heads=3),
    "page_1": dict(new=[9, 20], ctx=[3, 0], page=1, dim=32),
    "page_5": dict(new=[9, 20], ctx=[3, 0], page=5, dim=96, heads=1),
    "wide": dict(new=[21], ctx=[4], dim=256, heads=5),
    "d192": dict(new=[21], ctx=[4], dim=192, page=24),
    "d128": dict(new=[50, 2], ctx=[4, 100], dim=128, heads=8, layers=3),
}


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("name", CASES)
def test_append_quantises(K, name, dtype):
    """Codes and scales as the definition has them; nothing else is written."""
    c = dict(CASES[name])
    p = Pool(K, **c)
    layer = p.cache.shape[0] - 1
    g = torch.Generator().manual_seed(3)
    heads = p.cache.shape[4]
    qkv = torch.randn((p.tokens, 4 * heads, p.dim), generator=g) * torch.exp(2 * torch.randn((p.tokens, 4 * heads, 1), generator=g))
    qkv = qkv.to(TORCH[dtype]).cuda()
    k, v = qkv[:, 2 * heads:3 * heads], qkv[:, 3 * heads:]       # slices of a fused projection
    append(K, p, k, v, layer)
    page, slot = p.where()
    want_c, want_s = p.before[0].cpu().clone(), p.before[1].cpu().clone()
    for kv, x in enumerate((k, v)):
        code, byte = ref.quantise(x.cpu())
        want_c[layer, kv][page, slot] = ref.pack(code)
        want_s[layer, kv][page, slot] = byte.to(torch.uint8)
    assert torch.equal(p.scales.cpu(), want_s)
    assert torch.equal(p.cache.cpu(), want_c)


def test_every_value(K):
    """All finite 16-bit values beside group maxima near every border of a scale, exactly."""
    for dtype in (torch.bfloat16, torch.float16):
        bits = torch.arange(0, 65536, dtype=torch.int32).to(torch.int16).view(dtype)
        x = bits[torch.isfinite(bits)].float()
        top = (x.abs() * torch.tensor([1.0, 1.75, 1.7578125, 3.5])[torch.arange(len(x)) % 4]).to(dtype)
        top = torch.where(torch.isfinite(top), top, x.to(dtype))
        rows = torch.zeros((len(x), 32), dtype=dtype)
        rows[:, 5], rows[:, 17] = x.to(dtype), top
        rows[:, 9] = (x * 0.625).to(dtype)
        n = len(x) // 4 * 4
        rows = rows[:n].view(n // 4, 1, 128).cuda()
        p = Pool(K, [n // 4], [0], heads=1, dim=128)
        append(K, p, rows, rows)
        page, slot = p.where()
        code, byte = ref.quantise(rows.cpu())
        assert torch.equal(p.scales.cpu()[0, 1][page, slot], byte.to(torch.uint8))
        assert torch.equal(p.cache.cpu()[0, 0][page, slot], ref.pack(code))


def test_error_is_half_a_step(K):
    """No element is off by more than half a step of its size: 2^-2 of it, or a quarter of the scale."""
    p = Pool(K, [64], [0], heads=2, dim=128)
    x = torch.randn((64, 2, 128), generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    append(K, p, x, x)
    k, v = torch.empty_like(x), torch.empty_like(x)
    K.kvx_fetch(p.view, p.batch, 0, k, v)
    assert torch.equal(k, v)
    x, y = x.double().cpu(), k.double().cpu()
    unit = (2.0 ** (ref.quantise(x)[1].double() - 127)).repeat_interleave(32, -1)
    assert ((x - y).abs() <= torch.maximum(x.abs() / 4, unit / 4)).all()


def test_not_finite(K):
    """A group with a NaN or an infinity reads as NaN; the other groups of the row are what they are."""
    x = torch.randn((6, 2, 96), generator=torch.Generator().manual_seed(2)).bfloat16()
    x[0, 0, 3], x[1, 1, 40], x[2, 0, 95], x[3, 1, 64] = math.nan, math.inf, -math.inf, math.nan
    x[4] = 0.0
    p = Pool(K, [6], [10], heads=2, dim=96)
    append(K, p, x.cuda(), x.cuda())
    k, v = torch.empty_like(x).cuda(), torch.empty_like(x).cuda()
    K.kvx_fetch(p.view, p.batch, 0, k, v)
    want = ref.dequantise(*ref.quantise(x))
    got = k.double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.isnan(want).sum() == 4 * 32
    assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want)) and (got[4] == 0).all()


def test_largest_values(K):
    """The scale is cut where the largest code would be infinite, and at the smallest normal."""
    x = torch.zeros((2, 1, 32), dtype=torch.bfloat16)
    x[0, 0, :3] = torch.tensor([3.38e38, -3.0e38, 1.0e38])
    x[1, 0, :3] = torch.tensor([1e-40, 3e-39, -1e-38])
    p = Pool(K, [2], [0], heads=1, dim=32)
    append(K, p, x.cuda(), x.cuda())
    code, byte = ref.quantise(x)
    page, slot = p.where()
    assert byte[:, 0, 0].tolist() == [252, 1]
    assert torch.equal(p.scales.cpu()[0, 0][page, slot], byte.to(torch.uint8))
    assert torch.equal(p.cache.cpu()[0, 0][page, slot], ref.pack(code))


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("pairs", [32, 20])
def test_append_turns_and_quantises(K, interleaved, pairs):
    """Rotary positions first: a turned value is off by less than 2^-20 of its pair, which may pass
    one border of the code."""
    p = Pool(K, [40, 7], [100, 0], heads=2, dim=64)
    g = torch.Generator().manual_seed(5)
    k, v = (torch.randn((47, 2, 64), generator=g).bfloat16() for _ in range(2))
    q = torch.randn((47, 4, 64), generator=g).bfloat16()
    inv = 10000.0 ** (-torch.arange(pairs, dtype=torch.float32) / pairs)
    pos = torch.randint(0, 5000, (1, 47), generator=g, dtype=torch.int32)
    q_out = torch.empty_like(q).cuda()
    K.kvx_append(p.view, p.batch, K.make_rope(inv.cuda(), [pairs], pos.cuda(), interleaved=interleaved), 0, q.cuda(),
                 k.cuda(), v.cuda(), q_out)
    turned = ops.rotate(k, inv, [pairs], pos, interleaved)
    page, slot = p.where()
    got = ref.dequantise(ref.unpack(p.cache.cpu()[0, 0][page, slot]), p.scales.cpu()[0, 0][page, slot])
    code, byte = ref.quantise(turned)
    want = ref.dequantise(code, byte)
    unit = (2.0 ** (byte.double() - 127)).repeat_interleave(32, -1)
    size = turned.abs().amax(-1, keepdim=True)
    # a border is passed only by values that lie next to one
    border = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], dtype=torch.float64)
    near = ((turned.abs() / unit)[..., None] - border).abs().amin(-1) * unit <= size * 2.0 ** -19
    near[..., 2 * pairs:] = False        # what is not turned is exact, on a border too (16-bit values often are)
    top = turned.unflatten(-1, (-1, 32)).abs().amax(-1)
    edge = ((torch.frexp(top)[0] - 0.875).abs() < 2.0 ** -18).repeat_interleave(32, -1)
    assert ((got == want) | near | edge).all()
    assert near.float().mean() < 0.001
    back = ref.dequantise(ref.unpack(p.cache.cpu()[0, 1][page, slot]), p.scales.cpu()[0, 1][page, slot])
    assert torch.equal(back, ref.dequantise(*ref.quantise(v)))
    want_q = ops.rotate(q, inv, [pairs], pos, interleaved)
    assert ((q_out.double().cpu() - want_q).abs() <= want_q.abs() * 2.0 ** -8 + 2.0 ** -18 * q.abs().max()).all()


def stored(p, layer, kv):
    """The batch's rows as they lie in the cache, float64."""
    page, slot = p.where()
    if p.kind == "e2m1":
        return ref.dequantise(ref.unpack(p.cache.cpu()[layer, kv][page, slot]), p.scales.cpu()[layer, kv][page, slot])
    bits = p.cache.cpu().view(torch.uint8 if p.scales is not None else torch.int16)[layer, kv][page, slot]
    x = bits.view(p.cache.dtype).double()
    return x if p.scales is None else (x.float() * p.scales.cpu()[layer, kv][page, slot][..., None]).double()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("kind", ["e2m1", "e4m3fn", "e5m2", "bf16", "fp16"])
@pytest.mark.parametrize("name", CASES)
def test_fetch(K, name, kind, dtype):
    """Every code (the pools are random bytes), to the nearest of the 16-bit type, bit for bit."""
    p = Pool(K, kind=kind, **CASES[name])
    layer, heads = p.cache.shape[0] - 1, p.cache.shape[4]
    out = torch.full((p.tokens + 1, 3 * heads, p.dim), 7.0, dtype=TORCH[dtype], device="cuda")
    K.kvx_fetch(p.view, p.batch, layer, out[:-1, :heads], out[:-1, 2 * heads:])
    for kv, part in enumerate((out[:-1, :heads], out[:-1, 2 * heads:])):
        want = stored(p, layer, kv).to(TORCH[dtype])
        got = part.cpu()
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        ok = ~torch.isnan(want)
        assert torch.equal(got[ok], want[ok])
    assert (out[:, heads:2 * heads] == 7.0).all() and (out[-1] == 7.0).all()
    assert torch.equal(p.cache.view(torch.uint8), p.before[0].view(torch.uint8))


@pytest.mark.parametrize("byte", [0, 1, 100, 127, 252, 253, 254, 255])
def test_scale_bytes(K, byte):
    """What a scale byte stands for, at the ends of the range; above 252 it is no number."""
    p = Pool(K, [4], [0], heads=1, dim=32)
    p.scales.fill_(byte)
    k, v = (torch.empty((4, 1, 32), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    K.kvx_fetch(p.view, p.batch, 0, k, v)
    want = stored(p, 0, 0).to(torch.bfloat16)
    if byte > 252:
        assert torch.isnan(k).all()
    else:
        assert torch.equal(k.cpu(), want)


def test_pages_that_are_none(K):
    """Rows of pages outside the pool are not written, and read as zeros."""
    p = Pool(K, [40], [0], heads=2, dim=64)
    table = p.table.clone()
    table[0, 1], table[0, 2] = -1, p.blocks
    view = K.make_cache(p.cache, p.scales, table.cuda(), dtype=K.E2M1)
    x = torch.randn((40, 2, 64), generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    K.kvx_append(view, p.batch, no_rope(K, 40), 0, None, x, x, None)
    k, v = torch.full_like(x, 9.0), torch.full_like(x, 9.0)
    K.kvx_fetch(view, p.batch, 0, k, v)
    want = ref.dequantise(*ref.quantise(x.cpu()))
    assert torch.equal(k[:16].double().cpu(), want[:16]) and (k[16:] == 0).all() and (v[16:] == 0).all()
    page, slot = p.where()
    assert torch.equal(p.cache[0, :, page[16:], slot[16:]], p.before[0][0, :, page[16:], slot[16:]])


def test_bounds_cut(K):
    """Lengths on the device beyond the host's bounds: what lies past them reads as zeros, tokens of no
    request are left as they were."""
    p = Pool(K, [20, 20], [0, 0], heads=1, dim=64)
    batch = K.make_batch(int32([0, 20, 30]), int32([0, 0]), 40, 12, 10)
    k, v = (torch.full((40, 1, 64), 9.0, dtype=torch.float16, device="cuda") for _ in range(2))
    K.kvx_fetch(p.view, batch, 0, k, v)
    want = stored(p, 0, 0).to(torch.float16)
    assert torch.equal(k[:10].cpu(), want[:10]) and (k[10:20] == 0).all()
    assert torch.equal(k[20:30].cpu(), want[20:30]) and (k[30:] == 9.0).all()


@pytest.mark.parametrize("heads,dim", [(1, 32), (2, 64), (3, 96), (8, 128), (5, 256)])
def test_commit_moves_rows(K, heads, dim):
    p = Pool(K, [9, 30, 0, 5], [13, 0, 4, 31], heads=heads, dim=dim, layers=3)
    accepted = [[0, 2, 5, 8], [1, 4, 9, 29], [0, 1, 2, 3], [0, 1, 2, 4]]
    counts = [4, 3, 0, 4]
    new_lens = torch.empty(4, dtype=torch.int32, device="cuda")
    K.kvx_commit(p.view, 0, 3, int32(p.ctx), int32(accepted), int32(counts), new_lens)
    want_c, want_s = p.before[0].cpu().clone(), p.before[1].cpu().clone()
    for r, n in enumerate(counts):
        for i in range(n):
            a, b = (p.ctx[r] + accepted[r][i], p.ctx[r] + i)
            pa, pb = (int(p.table[r, x // 16]) for x in (a, b))
            for w, src in ((want_c, p.before[0].cpu()), (want_s, p.before[1].cpu())):
                w[:, :, pb, b % 16] = src[:, :, pa, a % 16]
    assert torch.equal(p.cache.cpu(), want_c) and torch.equal(p.scales.cpu(), want_s)
    assert new_lens.tolist() == [c + n for c, n in zip(p.ctx, counts)]


@pytest.mark.parametrize("heads,dim", [(1, 32), (2, 64), (3, 96), (2, 128), (1, 256)])
def test_evict_moves_rows(K, heads, dim):
    p = Pool(K, [0, 0, 0], [100, 30, 260], heads=heads, dim=dim, layers=2)
    g = torch.Generator().manual_seed(8)
    w = torch.rand((2, 3, heads, 260), generator=g)
    budget, sink, recent = 64, 4, 16
    kept = torch.empty((2, 3, heads, budget), dtype=torch.int32, device="cuda")
    lens = torch.empty(3, dtype=torch.int32, device="cuda")
    dw = w.cuda()
    K.kvx_evict(p.view, 0, 2, int32(p.ctx), 260, budget, sink, recent, dw, dw, kept, lens)
    want_c, want_s = p.before[0].cpu().clone(), p.before[1].cpu().clone()
    for layer in range(2):
        for r in range(3):
            for h in range(heads):
                stay = ops.evict(p.ctx[r], budget, sink, recent, w[layer, r, h])
                for i, j in enumerate(stay):
                    a, b = int(p.table[r, j // 16]), int(p.table[r, i // 16])
                    for x, src in ((want_c, p.before[0].cpu()), (want_s, p.before[1].cpu())):
                        x[layer, :, b, i % 16, h] = src[layer, :, a, j % 16, h]
    assert torch.equal(p.cache.cpu(), want_c) and torch.equal(p.scales.cpu(), want_s)


def test_offsets_past_32_bits(K):
    """A pool whose rows lie past 2^32 bytes and its scale bytes past 2^31: pages at its end."""
    blocks, page, heads, dim = 2 ** 19, 16, 8, 256          # 2 x 8.6 GB
    cache = torch.zeros((1, 2, blocks, page, heads, dim // 2), dtype=torch.uint8, device="cuda")
    scales = torch.full((1, 2, blocks, page, heads, dim // 32), 127, dtype=torch.uint8, device="cuda")
    table = int32([[blocks - 1, blocks // 2 + 3, 1]])
    view = K.make_cache(cache, scales, table, dtype=K.E2M1)
    batch = K.make_batch(int32([0, 40]), int32([0]), 40, 40, 40)
    x, y = (torch.randn((40, heads, dim), generator=torch.Generator().manual_seed(s)).bfloat16().cuda() for s in (1, 2))
    K.kvx_append(view, batch, no_rope(K, 40), 0, None, x, y, None)
    k, v = torch.empty_like(x), torch.empty_like(x)
    K.kvx_fetch(view, batch, 0, k, v)
    for got, src in ((k, x), (v, y)):
        assert torch.equal(got.double().cpu(), ref.dequantise(*ref.quantise(src.cpu())))
    code, byte = ref.quantise(y[:16].cpu())
    assert torch.equal(cache[0, 1, blocks - 1].cpu(), ref.pack(code))
    assert torch.equal(scales[0, 1, blocks - 1].cpu(), byte.to(torch.uint8))


def test_captured(K):
    """Append and fetch in a graph that is replayed with other rows, another stream, eager work between."""
    p = Pool(K, [3, 5], [20, 0], heads=2, dim=128)
    g = torch.Generator().manual_seed(4)
    x = torch.zeros((8, 2, 128), dtype=torch.float16, device="cuda")
    k, v = torch.empty_like(x), torch.empty_like(x)
    rope = no_rope(K, 8)
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        K.kvx_append(p.view, p.batch, rope, 0, None, x, x, None, stream=stream)
        stream.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            K.kvx_append(p.view, p.batch, rope, 0, None, x, x, None, stream=stream)
            K.kvx_fetch(p.view, p.batch, 0, k, v, stream=stream)
    for _ in range(4):
        rows = torch.randn((8, 2, 128), generator=g).half()
        x.copy_(rows)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(k.double().cpu(), ref.dequantise(*ref.quantise(rows)))
        (k * 2).sum().item()
