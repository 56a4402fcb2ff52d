"""kvx_attend and kvx_weigh against the plain form in 64 bits: types, head
shapes, lengths from none to many, trees, masks that leave a row empty, windows,
prefixes, bias and capped scores; what a token does not see never counts."""
import math

import pytest
import torch

import operator_reference as ref
from operator_reference import UNIT, Problem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def K():
    import paper_2509_17542_amd as K
    return K


def run(K, p, stream=None, q=None):
    view, batch, scores = p.gpu(K)
    q = p.q.cuda() if q is None else q
    out = torch.full((p.tokens, p.q_heads, p.dim), math.nan, dtype=p.q.dtype, device="cuda")
    lse = torch.full((p.tokens, p.q_heads), math.nan, dtype=torch.float32, device="cuda")
    nbytes = K.kvx_attend_workspace(view, batch, p.q_heads)
    ws = torch.full((max(nbytes, 16),), 0xFF, dtype=torch.uint8, device="cuda")
    K.kvx_attend(view, batch, scores, p.layer, q, out, lse, ws, stream=stream)
    return out, lse, (view, batch, scores, ws)


def check(p, out, lse):
    """Weights and the output are rounded once each to 16 bits (a weight also to
    the power of two of its row's reference, no further than u), on top of the
    scores' error, which acts on a weight twice: through it and through the sum."""
    want, z, size, delta = ref.attend(p)
    out, lse = out.double().cpu(), lse.double().cpu()
    u = UNIT[p.dtype]
    tol = size * (2.1 * u + 4 * delta[..., None] + 2.0 ** -18) + 2.0 ** -24
    assert torch.isfinite(out).all()
    bad = (out - want).abs() - tol
    assert bad.max() <= 0 if bad.numel() else True, f"out off by {(out - want).abs().max()}"
    empty = z == -math.inf
    assert torch.equal(lse == -math.inf, empty)
    assert (out[empty] == 0).all()
    e = (lse - z)[~empty].abs()
    assert (e <= (delta + 2.0 ** -21 * (1 + z.abs()))[~empty]).all(), f"lse off by {e.max()}"


TYPES = [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "e4m3fn"), ("fp16", "e4m3fn"), ("bf16", "e5m2"),
         ("fp16", "e5m2")]

CASES = {
    "one": dict(new=[1], ctx=[37]),
    "first": dict(new=[1], ctx=[0]),
    "lengths": dict(new=[1, 1, 1, 1, 1, 1], ctx=[0, 1, 15, 16, 31, 300]),
    "none_new": dict(new=[0, 1, 0, 2, 0], ctx=[5, 64, 0, 63, 9]),
    "long": dict(new=[1, 1], ctx=[2500, 1031], group=4),
    "two": dict(new=[2, 1], ctx=[129, 700], group=8),
    "tree": dict(new=[13, 7, 1], ctx=[65, 0, 200], tree=1, group=4),
    "tree_wide": dict(new=[64, 70, 33], ctx=[500, 17, 0], tree=2, group=2),
    "tree_many": dict(new=[200], ctx=[310], tree=3, group=7, heads=1),
    "chain": dict(new=[100, 33, 64], ctx=[0, 190, 64], group=4),
    "chain_long": dict(new=[300], ctx=[700], group=2),
    "chain_fresh": dict(new=[257, 128], ctx=[0, 0], group=1, heads=3),
    "capped": dict(new=[1, 9], ctx=[77, 205], softcap=20.0, tree=4, values=3.0),
    "bias": dict(new=[1, 9, 40], ctx=[77, 205, 12], slopes=True, tree=5, group=3),
    "bias_chain": dict(new=[50], ctx=[205], slopes=True, softcap=30.0),
    "window": dict(new=[1, 9, 70], ctx=[77, 205, 300], window=33),
    "window_tree": dict(new=[5, 30], ctx=[400, 205], window=16, tree=6, group=4),
    "window_prefix": dict(new=[1, 9, 70], ctx=[77, 205, 300], window=33, prefix=[4, 0, 80]),
    "window_one": dict(new=[1, 40], ctx=[77, 205], window=1),
    "prefix_ahead": dict(new=[60, 20], ctx=[0, 30], prefix=[25, 45]),
    "positions": dict(new=[4], ctx=[60], positions=[90, 75, 61, 60], slopes=True, window=30),
    "odd_group": dict(new=[1, 3], ctx=[100, 41], group=5, heads=3),
    "group_16": dict(new=[1, 2, 17], ctx=[300, 41, 100], group=16, heads=1),
    "group_40": dict(new=[1, 2], ctx=[300, 41], group=40, heads=2),
    "page_1": dict(new=[1, 20], ctx=[60, 41], page=1),
    "page_5": dict(new=[1, 20], ctx=[101, 41], page=5),
    "page_128": dict(new=[1, 20], ctx=[300, 141], page=128),
    "page_24": dict(new=[3, 150], ctx=[300, 141], page=24),
    "layer": dict(new=[1, 20], ctx=[60, 41], layers=3, layer=1),
    "large_scores": dict(new=[1, 20], ctx=[160, 41], values=12.0),
}


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("name", CASES)
def test_attend(K, name, dtype, cache):
    p = Problem(dtype=dtype, cache=cache, **CASES[name])
    out, lse, _ = run(K, p)
    check(p, out, lse)


@pytest.mark.parametrize("dim", [16, 48, 64, 80, 96, 112, 128, 144, 192, 208, 256])
@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("fp16", "e4m3fn")])
@pytest.mark.parametrize("shape", [dict(new=[1, 2], ctx=[200, 90]), dict(new=[40, 9], ctx=[200, 90], tree=9)])
def test_head_dims(K, dim, dtype, cache, shape):
    p = Problem(dim=dim, dtype=dtype, cache=cache, group=3, seed=dim, **shape)
    out, lse, _ = run(K, p)
    check(p, out, lse)


@pytest.mark.parametrize("dim", [16, 64, 80, 128, 256])
@pytest.mark.parametrize("shape", [dict(new=[1, 2, 1], ctx=[5 * 512 - 3, 700, 29 * 512]),
                                   dict(new=[1, 1], ctx=[33 * 512 + 7, 41 * 512]),
                                   dict(new=[37], ctx=[3 * 1024 + 5]),
                                   dict(new=[9, 20], ctx=[37 * 1024 + 11, 900], tree=3)], ids=str)
def test_splits(K, dim, shape):
    """Slots over several workgroups, a number of them that does not divide by the
    splits a wave joins at once, fewer and more than 32."""
    p = Problem(dim=dim, heads=1, group=5, seed=dim, **shape)
    out, lse, _ = run(K, p)
    check(p, out, lse)


@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "e4m3fn")])
def test_many_requests_of_few_rows(K, dtype, cache):
    """512 pairs of a request and a KV head, at most 20 rows each, many far fewer."""
    p = Problem(dim=64, heads=8, group=4, dtype=dtype, cache=cache, tree=2,
                new=[1 + r % 5 if r % 7 else 0 for r in range(64)], ctx=[(37 * r) % 211 for r in range(64)], seed=5)
    out, lse, _ = run(K, p)
    check(p, out, lse)


@pytest.mark.parametrize("ctx", [[219], [257], [700], [1500], [6001, 5]])
def test_short_calls_of_many_rows(K, ctx):
    """Few workgroups in all: slots cut finer than elsewhere, short requests idle."""
    p = Problem(dim=128, heads=1, group=4, dtype="fp16", cache="fp16", tree=4, new=[37, 12][:len(ctx)], ctx=ctx, seed=6)
    out, lse, _ = run(K, p)
    check(p, out, lse)


@pytest.mark.parametrize("dim", [8, 24, 72, 120, 200, 248])
def test_head_dims_of_8(K, dim):
    p = Problem(dim=dim, dtype="fp16", cache="fp16", new=[1, 19], ctx=[100, 50], seed=dim)
    out, lse, _ = run(K, p)
    check(p, out, lse)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("poison", [math.inf, -math.inf, math.nan])
def test_what_is_not_seen_never_counts(K, dtype, cache, poison):
    """Siblings of a tree, slots outside a window and later tokens hold
    infinities or NaN, in keys and values: rows that do not see them are as if
    they were not there."""
    for case in (dict(new=[3], ctx=[40], tree=3), dict(new=[20, 30], ctx=[40, 0], tree=7),
                 dict(new=[90], ctx=[40], tree=8, group=4)):
        p = Problem(dtype=dtype, cache=cache, **case)
        seen = {}
        for r, n in enumerate(p.new):
            # nodes that are nobody's ancestor but their own: poisoned, and their own rows left out
            for i in range(n):
                see, _ = p.sees(r, i)
                for j in torch.nonzero(see)[:, 0].tolist():
                    seen.setdefault((r, j), []).append(i)
        skip = []
        for r, n in enumerate(p.new):
            for i in range(n):
                if seen.get((r, p.ctx[r] + i)) == [i] and i % 2:
                    page, slot = p.slot(r, p.ctx[r] + i)
                    skip.append(p.starts[r] + i)
                    if p.scales is None:
                        p.cache[p.layer, :, page, slot] = poison
                    elif cache == "e5m2" and math.isinf(poison):
                        p.cache.view(torch.uint8)[p.layer, :, page, slot] = 0x7C if poison > 0 else 0xFC
                    elif math.isinf(poison):
                        p.scales[p.layer, :, page, slot] = poison
                    else:
                        p.cache.view(torch.uint8)[p.layer, :, page, slot] = 0x7F
        assert skip
        keep = [t for t in range(p.tokens) if t not in skip]
        out, lse, _ = run(K, p)
        want, z, size, delta = ref.attend(p)
        tol = (size * (2.1 * UNIT[dtype] + 4 * delta[..., None] + 2.0 ** -18) + 2.0 ** -24)[keep]
        assert ((out.double().cpu() - want)[keep].abs() <= tol).all()
        assert ((lse.double().cpu() - z)[keep].abs() <= (delta + 2.0 ** -21 * (1 + z.abs()))[keep]).all()


def test_infinite_values_that_are_seen(K):
    """An infinite value that a row sees gives that row an infinity, and only
    that row; opposite infinities give NaN."""
    for new, tree in ([3], 3), ([40], 8):
        p = Problem(new=new, ctx=[40], tree=tree, dtype="bf16", cache="bf16")
        n, c = new[0], 40
        page, slot = p.slot(0, c + 1)
        p.cache[0, 1, page, slot, :, 3] = math.inf
        page, slot = p.slot(0, c + 2)
        p.cache[0, 1, page, slot, :, 3] = -math.inf
        p.cache[0, 1, page, slot, :, 5] = math.nan
        out, _, _ = run(K, p)
        out = out.float().cpu()
        for i in range(n):
            see, _ = p.sees(0, i)
            up, down = bool(see[c + 1]), bool(see[c + 2])
            x = out[i, :, 3]
            if up and down:
                assert torch.isnan(x).all()
            elif up or down:
                assert (x == (math.inf if up else -math.inf)).all()
            else:
                assert torch.isfinite(x).all()
            assert torch.isnan(out[i, :, 5]).all() == down
            assert torch.isfinite(out[i, :, [0, 1, 2, 4, 6, 7]]).all()


def test_rows_that_see_nothing(K):
    """A tree bit of its own missing and no context: zeros and -infinity."""
    p = Problem(new=[3, 20, 1], ctx=[0, 0, 0], tree=1, group=3)
    p.tree[0] = 0
    p.tree[5] = 0
    p.tree[10] = 0
    p.tree[23] = 0
    out, lse, _ = run(K, p)
    check(p, out, lse)
    assert (lse[[0, 5, 10, 23]] == -math.inf).all() and (out[[0, 5, 10, 23]] == 0).all()


def test_pages_that_are_none(K):
    """A page id outside the pool hides its slots, in the middle too."""
    for new, ctx in ([1, 1], [100, 90]), ([30, 2], [100, 90]):
        p = Problem(new=new, ctx=ctx, group=4)
        p.table[0, 2] = -1
        p.table[1, 0] = p.blocks
        p.table[1, 3] = 2 ** 31 - 1
        out, lse, _ = run(K, p)
        check(p, out, lse)


def test_bounds_cut_lengths(K):
    """Lengths on the device above the host's bounds are cut to them."""
    p = Problem(new=[1, 1], ctx=[100, 40])
    view, batch, scores = p.gpu(K)
    big = torch.tensor([10 ** 6, 40], dtype=torch.int32).cuda()
    batch2 = K.make_batch(batch.keep[0], big, p.tokens, 1, 48)
    q, out = p.q.cuda(), torch.zeros_like(p.q, device="cuda")
    ws = torch.zeros(max(16, K.kvx_attend_workspace(view, batch2, p.q_heads)), dtype=torch.uint8, device="cuda")
    K.kvx_attend(view, batch2, scores, 0, q, out, None, ws)
    small = Problem(new=[1, 1], ctx=[100, 40])
    small.ctx, small.total = [48, 40], [48, 41]     # request 0: 48 slots, its own token cut off
    want, _, size, delta = ref.attend(small)
    tol = size * (2.1 * UNIT["bf16"] + 4 * delta[..., None] + 2.0 ** -18) + 2.0 ** -24
    assert ((out.double().cpu() - want).abs() <= tol).all()


def test_strided_rows(K):
    """q and out as slices of wider rows; what lies beside them is not written."""
    p = Problem(new=[2, 30], ctx=[100, 41], group=4)
    wide = torch.randn((p.tokens, p.q_heads + 6, p.dim), device="cuda").to(p.q.dtype)
    wide[:, 2:2 + p.q_heads] = p.q.cuda()
    view, batch, scores = p.gpu(K)
    store = torch.full((p.tokens, p.q_heads + 3, p.dim), 7.0, dtype=p.q.dtype, device="cuda")
    out = store[:, 1:1 + p.q_heads]
    ws = torch.zeros(max(16, K.kvx_attend_workspace(view, batch, p.q_heads)), dtype=torch.uint8, device="cuda")
    lse = torch.zeros((p.tokens, p.q_heads), device="cuda")
    K.kvx_attend(view, batch, scores, 0, wide[:, 2:2 + p.q_heads], out, lse, ws)
    check(p, out, lse)
    assert (store[:, 0] == 7).all() and (store[:, 1 + p.q_heads:] == 7).all()


def test_another_stream_and_repeats(K):
    """On a stream of its own, the same bits every time."""
    p = Problem(new=[1, 30], ctx=[900, 400], group=4, dim=128)
    s = torch.cuda.Stream()
    first, lse, _ = run(K, p)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        again, lse2, keep = run(K, p)
        third, lse3, keep3 = run(K, p, stream=s)
    s.synchronize()
    assert torch.equal(first, again) and torch.equal(lse, lse2)
    assert torch.equal(first, third) and torch.equal(lse, lse3)


def test_graph_follows_the_lengths(K):
    """Recorded once, replayed with other lengths, tokens and tables in the same buffers."""
    a = Problem(new=[1, 5], ctx=[300, 100], group=4, seed=1, blocks=60)
    b = Problem(new=[2, 4], ctx=[17, 290], group=4, seed=2, blocks=60)
    for p in (a, b):
        p.max_context, p.max_tokens = 320, 6
        table = torch.full((2, 21), -1, dtype=torch.int32)
        table[:, :p.table.shape[1]] = p.table
        p.table = table
    view, batch, scores = a.gpu(K)
    q = a.q.cuda()
    out, lse = torch.zeros_like(q), torch.zeros((6, a.q_heads), device="cuda")
    ws = torch.zeros(max(16, K.kvx_attend_workspace(view, batch, a.q_heads)), dtype=torch.uint8, device="cuda")
    K.kvx_attend(view, batch, scores, 0, q, out, lse, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        K.kvx_attend(view, batch, scores, 0, q, out, lse, ws)
    for p in (a, b, a, b):
        view.keep[0].view(torch.int16).copy_(p.cache.view(torch.int16))
        view.keep[2].copy_(p.table)
        batch.keep[0].copy_(torch.tensor(p.starts, dtype=torch.int32))
        batch.keep[1].copy_(torch.tensor(p.ctx, dtype=torch.int32))
        q.copy_(p.q)
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        check(p, out, lse)


def test_offsets_past_32_bits(K):
    """Pages whose bytes and elements lie past 2^32 of their plane."""
    page, heads, dim = 64, 8, 128
    blocks = 2 ** 33 // (page * heads * dim) // 2 + 64        # 2^32 elements and more a plane
    cache = torch.empty((1, 2, blocks, page, heads, dim), dtype=torch.bfloat16, device="cuda")
    p = Problem(new=[1, 20], ctx=[100, 300], heads=heads, group=2, dim=dim, page=page)
    moved = p.table.clone()
    used = sorted(set(p.table[p.table >= 0].tolist()))
    for n, b in enumerate(used):
        to = blocks - 1 - n
        cache[0, :, to] = p.cache[0, :, b].cuda()
        moved[p.table == b] = to
    view, batch, scores = p.gpu(K)
    view = K.make_cache(cache, None, moved.cuda())
    q, out = p.q.cuda(), torch.zeros_like(p.q, device="cuda")
    lse = torch.zeros((p.tokens, p.q_heads), device="cuda")
    ws = torch.zeros(max(16, K.kvx_attend_workspace(view, batch, p.q_heads)), dtype=torch.uint8, device="cuda")
    K.kvx_attend(view, batch, scores, 0, q, out, lse, ws)
    check(p, out, lse)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("name", CASES)
def test_weigh(K, name, dtype, cache):
    p = Problem(dtype=dtype, cache=cache, **CASES[name])
    view, batch, scores = p.gpu(K)
    _, z, _, _ = ref.attend(p)
    lse = z.float().cuda()
    start = torch.rand((len(p.new), p.heads, p.max_context + 3))
    w = start.cuda()
    K.kvx_weigh(view, batch, scores, p.layer, p.q.cuda(), lse, w)
    want, tol = ref.weigh(p, lse.cpu(), start)
    got = w.double().cpu()
    assert ((got - want).abs() <= tol).all(), (got - want).abs().max()
    for r, t in enumerate(p.total):
        assert torch.equal(w[r, :, t:].cpu(), start[r, :, t:])


def test_weigh_what_is_not_seen(K):
    """NaN in keys that a row does not see weigh nothing for it; a row that saw
    nothing weighs nothing; a page that is none weighs 0."""
    p = Problem(new=[30], ctx=[100], tree=5, group=3)
    p.table[0, 2] = -1
    page, slot = p.slot(0, 100 + 29)
    p.cache[0, 0, page, slot] = math.nan
    for i in range(30):
        p.tree[i, 0] &= ~(1 << 29)
    view, batch, scores = p.gpu(K)
    _, z, _, _ = ref.attend(p)
    z[3] = -math.inf
    w = torch.full((1, p.heads, p.max_context), 0.5, device="cuda")
    K.kvx_weigh(view, batch, scores, 0, p.q.cuda(), z.float().cuda(), w)
    want, tol = ref.weigh(p, z.float(), torch.full((1, p.heads, p.max_context), 0.5))
    assert ((w.double().cpu() - want).abs() <= tol).all()
    assert (w[0, :, 129] == 0).all() and (w[0, :, 32:48] == 0.5).all()
