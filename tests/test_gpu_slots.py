"""kvx_append, kvx_evict and kvx_commit against the plain forms."""
import math
import random

import pytest
import torch

import operator_reference as ref
from operator_reference import FMAX, TORCH, UNIT, Problem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def K():
    import paper_2509_17542_amd as K
    return K


def bits(x):
    return x.view(torch.int32 if x.element_size() == 4 else
                  torch.int16 if x.element_size() == 2 else torch.uint8)


# ---- append ------------------------------------------------------------------

ROPES = {
    "halves": dict(sections=[32], interleaved=False),
    "interleaved": dict(sections=[32], interleaved=True),
    "axes": dict(sections=[8, 12, 12], interleaved=False),
    "axes4": dict(sections=[5, 0, 20, 7], interleaved=True),
    "partial": dict(sections=[16], interleaved=False),
    "partial_odd": dict(sections=[5, 6], interleaved=False),
    "partial_interleaved": dict(sections=[13], interleaved=True),
    "none": dict(sections=[0], interleaved=False),
}


def append(K, p, sections, interleaved, seed=0, top=5000, q_out=None, values=1.0):
    g = torch.Generator().manual_seed(seed)
    pairs = sum(sections)
    inv_freq = 10000.0 ** (-torch.arange(pairs, dtype=torch.float32) / max(pairs, 1))
    positions = torch.randint(0, top, (len(sections), p.tokens), generator=g, dtype=torch.int32)
    width = p.q_heads + 2 * p.heads
    qkv = (torch.randn((p.tokens, width, p.dim), generator=g) * values).to(TORCH[p.dtype])
    d = qkv.cuda()
    q, k, v = d.split([p.q_heads, p.heads, p.heads], dim=1)
    view, batch, _ = p.gpu(K)
    out = torch.zeros_like(q).contiguous() if q_out is None else q
    rope = K.make_rope(inv_freq.cuda(), sections, positions.cuda(), interleaved=interleaved)
    K.kvx_append(view, batch, rope, p.layer, q, k, v, out)
    torch.cuda.synchronize()
    hq, hk, hv = qkv.split([p.q_heads, p.heads, p.heads], dim=1)
    turn = [ref.rotate(x, inv_freq, sections, positions, interleaved) for x in (hq, hk)]
    return out, turn[0], (turn[1], hv.double()), (hq, hk, hv)


def check_append(p, out, want_q, want_kv):
    """One rounding to the target type on top of the fp32 turn (two products and
    a sum, each 2^-24 of the row's size, cosine and sine to 2^-22)."""
    slack = want_q.abs().amax(-1, keepdim=True) * 2.0 ** -20
    assert ((out.double().cpu() - want_q).abs() <= want_q.abs() * UNIT[p.dtype] + slack + 2.0 ** -25).all()
    got = p.d_cache.cpu()
    touched = torch.zeros(p.cache.shape[2:4], dtype=torch.bool)
    for r, n in enumerate(p.new):
        for i in range(n):
            page, slot = p.slot(r, p.ctx[r] + i)
            touched[page, slot] = True
            for kv in (0, 1):
                want = want_kv[kv][p.starts[r] + i]
                x = got[p.layer, kv, page, slot].double()
                big = want.abs().amax(-1)
                slack = big[:, None] * 2.0 ** -20
                if p.scales is None:
                    assert ((x - want).abs() <= want.abs() * UNIT[p.kind] + slack + 2.0 ** -25).all()
                else:
                    s = p.d_scales[p.layer, kv, page, slot].double().cpu()
                    assert ((s - big / FMAX[p.kind]).abs() <= s * 2.0 ** -19).all()
                    u, tiny = (2.0 ** -4, 2.0 ** -10) if p.kind == "e4m3fn" else (2.0 ** -3, 2.0 ** -17)
                    err = (x * s[:, None] - want).abs()
                    assert (err <= want.abs() * u * 1.001 + s[:, None] * tiny * 1.001 + slack).all()
    same = bits(got) == bits(p.cache)
    assert same[:, :, ~touched].all()
    other = [layer for layer in range(p.layers) if layer != p.layer]
    assert same[other].all()
    if p.scales is not None:
        same = bits(p.d_scales.cpu()) == bits(p.scales)
        assert same[:, :, ~touched].all() and same[other].all()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("cache", ["bf16", "fp16", "e4m3fn", "e5m2"])
@pytest.mark.parametrize("rope", ROPES)
def test_append(K, rope, dtype, cache):
    p = Problem(new=[3, 0, 1, 20], ctx=[0, 7, 33, 15], dtype=dtype, cache=cache, group=3)
    out, q, kv, _ = append(K, p, **ROPES[rope])
    check_append(p, out, q, kv)


@pytest.mark.parametrize("dim", [16, 48, 80, 112, 128, 192, 256])
@pytest.mark.parametrize("cache", ["bf16", "e4m3fn"])
def test_append_head_dims(K, dim, cache):
    p = Problem(new=[3, 20], ctx=[0, 15], cache=cache, dim=dim, layers=2, layer=1, page=5)
    out, q, kv, _ = append(K, p, [dim // 2 - 3, 3], False, seed=dim)
    check_append(p, out, q, kv)


def test_append_head_dims_of_8(K):
    for dim in (8, 24, 72, 248):
        p = Problem(new=[3, 20], ctx=[0, 15], cache="fp16", dtype="fp16", dim=dim)
        out, q, kv, _ = append(K, p, [dim // 2], True, seed=dim)
        check_append(p, out, q, kv)


def test_append_far_positions_and_in_place(K):
    """Angles of a million radians, q turned in place."""
    p = Problem(new=[40], ctx=[3], heads=4, group=4, dim=128)
    out, q, kv, _ = append(K, p, [64], False, top=1 << 20, q_out="q")
    check_append(p, out, q, kv)


def test_append_keys_and_values_only(K):
    p = Problem(new=[4, 1], ctx=[3, 70], cache="e4m3fn")
    k = torch.randn((5, 2, 64), device="cuda").bfloat16()
    v = torch.randn((5, 2, 64), device="cuda").bfloat16()
    view, batch, _ = p.gpu(K)
    rope = K.make_rope(torch.zeros(0, device="cuda"), [0], torch.zeros((1, 5), dtype=torch.int32, device="cuda"))
    K.kvx_append(view, batch, rope, 0, None, k, v, None)
    want = (k.double().cpu(), v.double().cpu())
    check_append(p, torch.zeros(0, 1, 64), torch.zeros((0, 1, 64), dtype=torch.float64), want)


def test_append_without_a_page(K):
    """A token whose slot has no page writes nothing; its query still turns."""
    p = Problem(new=[20, 4], ctx=[10, 0], spare=0)
    p.table[0, 1] = -1
    p.table[1, 0] = p.blocks
    out, q, kv, _ = append(K, p, [32], False)
    assert ((out.double().cpu() - q).abs() <= q.abs() * UNIT["bf16"] + 2.0 ** -17).all()
    got = p.d_cache.cpu()
    touched = torch.zeros(p.cache.shape[2:4], dtype=torch.bool)
    touched[p.table[0, 0], 10:] = True
    assert (bits(got) == bits(p.cache))[:, :, ~touched].all()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("cache", ["bf16", "fp16", "e4m3fn", "e5m2"])
def test_append_casts_as_the_conversion_does(K, dtype, cache):
    """Unturned rows land with the bits that kvx_repack gives them, infinities,
    NaN, zero rows and tiny rows among them."""
    heads, dim, page, n = 3, 64, 16, 37
    g = torch.Generator().manual_seed(5)
    x = torch.randn((1, 2, n, heads, dim), generator=g)
    x *= 10.0 ** (6 * torch.rand((1, 2, n, heads, 1), generator=g) - 4)
    x[0, 0, 1] = 0.0
    x[0, 1, 2, 1] = -0.0
    x[0, 0, 3, 0, 5] = math.nan
    x[0, 0, 4, 1, 9] = math.inf
    x[0, 1, 4, 2, 11] = -math.inf
    x[0, 1, 5, 0, :] = 1e-7
    x[0, 1, 6, 0, 3] = -math.nan
    src = x.to(TORCH[dtype]).cuda()
    f = {"fp16": K.FP16, "bf16": K.BF16, "e4m3fn": K.E4M3FN, "e5m2": K.E5M2}
    table = torch.tensor([[2, 0, 3]], dtype=torch.int32).cuda()
    shape = (1, 2, 4, page, heads, dim)
    caches = [torch.zeros(shape, dtype=TORCH[cache], device="cuda") for _ in range(2)]
    scales = [torch.zeros(shape[:-1], device="cuda") if cache in FMAX else None for _ in range(2)]
    plan = K.kvx_plan(K.make_desc(1, heads, dim, 1, 1, 0, f[dtype], f[cache], K.THD, page, 4, [n]))
    K.kvx_repack(plan, [src], caches[0], scales[0], table, 3)
    view = K.make_cache(caches[1], scales[1], table)
    ints = lambda v: torch.tensor(v, dtype=torch.int32).cuda()  # noqa: E731
    batch = K.make_batch(ints([0, n]), ints([0]), n, n, n)
    rope = K.make_rope(torch.zeros(0, device="cuda"), [0], torch.zeros((1, n), dtype=torch.int32, device="cuda"))
    K.kvx_append(view, batch, rope, 0, None, src[0, 0], src[0, 1], None)
    a, b = caches
    nan = torch.isnan(a.float())
    assert torch.equal(nan, torch.isnan(b.float()))
    assert (bits(a) == bits(b))[~nan].all()
    if cache in FMAX:
        assert torch.equal(bits(a), bits(b))
        assert torch.equal(bits(scales[0]), bits(scales[1]))


# ---- evict -------------------------------------------------------------------

def evict_case(K, lens, budget, sink, recent, heads=2, dim=64, cache="bf16", page=16, layers=2,
               weights=None, seed=0, in_place=False, layer0=0, all_layers=None):
    total = all_layers or layers
    p = Problem(new=[0] * len(lens), ctx=list(lens), heads=heads, dim=dim, cache=cache, dtype="bf16",
                page=page, layers=total, seed=seed)
    view, _, _ = p.gpu(K)
    g = torch.Generator().manual_seed(seed + 1)
    stride = max(max(lens), 1) + 5
    w = torch.rand((layers, len(lens), heads, stride), generator=g) if weights is None else weights
    d = w.cuda()
    w_out = d if in_place else torch.full_like(d, -5.0)
    kept = torch.full((layers, len(lens), heads, budget), -9, dtype=torch.int32, device="cuda")
    new_lens = torch.zeros(len(lens), dtype=torch.int32, device="cuda")
    K.kvx_evict(view, layer0, layers, torch.tensor(lens, dtype=torch.int32).cuda(), max(max(lens), 1), budget,
                sink, recent, d, w_out, kept, new_lens)
    torch.cuda.synchronize()
    assert new_lens.tolist() == [min(t, budget) for t in lens]
    want = bits(p.cache).clone()
    want_s = p.scales.clone() if p.scales is not None else None
    start, start_s = bits(p.cache), p.scales
    w_out, kept = w_out.cpu(), kept.cpu()
    for layer in range(layers):
        for r, T in enumerate(lens):
            for h in range(heads):
                stay = ref.evict(T, budget, sink, recent, w[layer, r, h].tolist())
                n = len(stay)
                assert kept[layer, r, h].tolist() == stay + [-1] * (budget - n), (layer, r, h)
                a, b = w_out[layer, r, h, :n], w[layer, r, h][stay]
                assert torch.equal(bits(a), bits(b))
                rest = w[layer, r, h, n:] if in_place else torch.full((stride - n,), -5.0)
                assert torch.equal(bits(w_out[layer, r, h, n:]), bits(rest))
                for i, j in enumerate(stay):
                    (pi, si), (pj, sj) = p.slot(r, i), p.slot(r, j)
                    if not (0 <= pi < p.blocks and 0 <= pj < p.blocks):
                        continue
                    want[layer0 + layer, :, pi, si, h] = start[layer0 + layer, :, pj, sj, h]
                    if want_s is not None:
                        want_s[layer0 + layer, :, pi, si, h] = start_s[layer0 + layer, :, pj, sj, h]
    assert torch.equal(bits(p.d_cache).cpu(), want)
    if want_s is not None:
        assert torch.equal(bits(p.d_scales).cpu(), bits(want_s))


@pytest.mark.parametrize("cache", ["bf16", "e4m3fn"])
@pytest.mark.parametrize("case", [
    dict(lens=[40, 0, 7, 33, 8, 1], budget=8, sink=1, recent=3),
    dict(lens=[300, 257, 256, 255], budget=256, sink=4, recent=32),
    dict(lens=[600], budget=64, sink=0, recent=0),
    dict(lens=[600, 100], budget=64, sink=64, recent=0),
    dict(lens=[600, 100], budget=64, sink=0, recent=64),
    dict(lens=[600, 100], budget=64, sink=30, recent=34),
    dict(lens=[1500, 900], budget=700, sink=4, recent=128, page=5),
    dict(lens=[20], budget=1, sink=0, recent=0, page=1),
    dict(lens=[5, 6], budget=100, sink=2, recent=2),
])
def test_evict(K, case, cache):
    evict_case(K, cache=cache, **case)
    evict_case(K, cache=cache, in_place=True, seed=3, **case)


@pytest.mark.parametrize("dim,cache", [(8, "fp16"), (80, "bf16"), (112, "e5m2"), (192, "e4m3fn"), (256, "bf16")])
def test_evict_head_dims(K, dim, cache):
    evict_case(K, [70, 33], 30, 2, 5, heads=3, dim=dim, cache=cache, layers=2, layer0=1, all_layers=4)


def test_evict_ties_and_odd_weights(K):
    """Equal weights: the lowest slots stay.  Zeros of both signs are equal, NaN
    is above infinity, negative weights have their order."""
    g = torch.Generator().manual_seed(0)
    pick = torch.tensor([0.0, -0.0, 1.0, 1.0, 2.0, math.inf, math.nan, -math.inf, -1.0, 1e-42, -1e-42, -math.nan])
    for seed in range(3):
        w = pick[torch.randint(0, len(pick), (2, 2, 2, 405), generator=g)]
        evict_case(K, [400, 390], 100 + 70 * seed, 2, 10, weights=w, seed=seed)
    evict_case(K, [400, 390], 100, 2, 10, weights=torch.zeros((2, 2, 2, 405)))
    evict_case(K, [400, 390], 100, 2, 10, weights=torch.full((2, 2, 2, 405), math.nan))


def test_evict_long(K):
    """More slots than a workgroup holds at once, weights close to each other."""
    g = torch.Generator().manual_seed(0)
    w = 1.0 + torch.randint(0, 3000, (1, 1, 1, 20005), generator=g) * 2.0 ** -23
    evict_case(K, [20000], 3000 + 71, 4, 100, heads=1, dim=16, layers=1, weights=w)


# ---- commit ------------------------------------------------------------------

@pytest.mark.parametrize("cache,dim", [("bf16", 64), ("e4m3fn", 128), ("e5m2", 80), ("fp16", 8)])
@pytest.mark.parametrize("page", [1, 5, 16])
def test_commit(K, cache, dim, page):
    new, ctx = [30, 5, 1, 64, 9, 12], [0, 17, 3, 100, 31, 16]
    p = Problem(new=new, ctx=ctx, cache=cache, dim=dim, page=page, layers=3, heads=3, dtype="bf16" if cache != "fp16" else "fp16")
    rnd = random.Random(page)
    paths = [sorted(rnd.sample(range(n), min(n, 7))) for n in new]
    paths[1] = []
    paths[4] = list(range(7))
    counts = [len(x) for x in paths]
    paths[5] = [2, 5, 5, 8, 9]                # ends at the entry that does not ascend
    counts[5] = 5
    accepted = torch.zeros((len(new), 7), dtype=torch.int32)
    for r, x in enumerate(paths):
        accepted[r, :len(x)] = torch.tensor(x, dtype=torch.int32)
    paths[5] = [2, 5]
    counts[3] = 100                           # cut to the stride
    view, _, _ = p.gpu(K)
    ints = lambda v: torch.tensor(v, dtype=torch.int32).cuda()  # noqa: E731
    new_lens = torch.zeros(len(new), dtype=torch.int32, device="cuda")
    K.kvx_commit(view, 1, 2, ints(ctx), accepted.cuda(), ints(counts), new_lens)
    torch.cuda.synchronize()
    assert new_lens.tolist() == [c + len(x) for c, x in zip(ctx, paths)]
    want, start = bits(p.cache).clone(), bits(p.cache)
    want_s = p.scales.clone() if p.scales is not None else None
    for r, x in enumerate(paths):
        for i, j in enumerate(x):
            (pi, si), (pj, sj) = p.slot(r, ctx[r] + i), p.slot(r, ctx[r] + j)
            want[1:, :, pi, si] = start[1:, :, pj, sj]
            if want_s is not None:
                want_s[1:, :, pi, si] = p.scales[1:, :, pj, sj]
    assert torch.equal(bits(p.d_cache).cpu(), want)
    if want_s is not None:
        assert torch.equal(bits(p.d_scales).cpu(), bits(want_s))


def test_commit_keeps_to_the_row(K):
    """Entries below 0 or past the block-table row end the path; a page that is
    none on either side leaves its row."""
    p = Problem(new=[20, 20, 20], ctx=[10, 10, 10], page=16)
    p.table[2, 1] = -1
    view, _, _ = p.gpu(K)
    ints = lambda v: torch.tensor(v, dtype=torch.int32).cuda()  # noqa: E731
    accepted = ints([[-1, 2, 3], [1, 2 ** 30, 2 ** 31 - 1], [2, 10, 11]])
    new_lens = torch.zeros(3, dtype=torch.int32, device="cuda")
    K.kvx_commit(view, 0, 1, ints([10, 10, 10]), accepted, ints([3, 3, 3]), new_lens)
    torch.cuda.synchronize()
    assert new_lens.tolist() == [10, 11, 13]
    want, start = bits(p.cache).clone(), bits(p.cache)
    for r, to, frm in ((1, 10, 11), (2, 10, 12)):
        (pi, si), (pj, sj) = p.slot(r, to), p.slot(r, frm)
        want[:, :, pi, si] = start[:, :, pj, sj]
    assert torch.equal(bits(p.d_cache).cpu(), want)
