"""kvx_attend over a 4-bit cache against the plain form in 64 bits, in the cases, with
the bounds and the poison of the other caches' tests; groups that are NaN, and the
calls that an engine makes."""
import math

import pytest
import torch

import operator_reference as ref
import serving_reference as four
from test_gpu_attend import CASES, check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def K():
    import paper_2509_17542_amd as K
    return K


class Problem(ref.Problem):
    """The same caches and batches, rows quantised to 4 bits; unused slots hold codes
    whose groups are NaN."""

    def __init__(self, *args, spread=0, **more):
        seed = more.get("seed", 0)
        super().__init__(*args, cache="bf16", poison=math.nan, **more)
        g = torch.Generator().manual_seed(seed + 99)
        x = self.cache.double()
        if spread:
            # rows' sizes apart by powers of two, outliers in a few of the groups
            x = x * 2.0 ** torch.randint(-spread, spread + 1, (*x.shape[:-1], 1), generator=g)
        code, byte = four.quantise(x)
        noise = torch.randint(0, 16, code.shape, generator=g)
        code = torch.where((byte > 252).repeat_interleave(32, -1), noise, code)
        self.codes, self.bytes = four.pack(code), byte.to(torch.uint8)

    def rows(self, kv, r):
        at = torch.arange(self.total[r])
        page = self.table[r].long()[at // self.page] if self.total[r] else at
        ok = (page >= 0) & (page < self.blocks)
        page = torch.where(ok, page, 0)
        x = four.dequantise(four.unpack(self.codes[self.layer, kv][page, at % self.page]),
                            self.bytes[self.layer, kv][page, at % self.page])
        return x, ok

    def gpu(self, K):
        cache = self.cache
        # the batch and the scores, over a stand-in for the cache that the others have
        self.cache = torch.zeros((1, 2, 1, 1, 1, 8), dtype=torch.bfloat16)
        _, batch, scores = super().gpu(K)
        self.cache = cache
        self.d_codes, self.d_bytes = self.codes.cuda(), self.bytes.cuda()
        view = K.make_cache(self.d_codes, self.d_bytes, self.table.cuda(), dtype=K.E2M1)
        return view, batch, scores


def run(K, p, stream=None, q=None, lse=True):
    view, batch, scores = p.gpu(K)
    q = p.q.cuda() if q is None else q
    out = torch.full((p.tokens, p.q_heads, p.dim), math.nan, dtype=p.q.dtype, device="cuda")
    z = torch.full((p.tokens, p.q_heads), math.nan, dtype=torch.float32, device="cuda") if lse else None
    nbytes = K.kvx_attend_workspace(view, batch, p.q_heads)
    ws = torch.full((max(nbytes, 16),), 0xFF, dtype=torch.uint8, device="cuda")
    K.kvx_attend(view, batch, scores, p.layer, q, out, z, ws, stream=stream)
    return out, z, (view, batch, scores, ws)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("name", CASES)
def test_attend(K, name, dtype):
    p = Problem(dtype=dtype, **CASES[name])
    out, lse, _ = run(K, p)
    check(p, out, lse)


@pytest.mark.parametrize("dim", [32, 64, 96, 128, 160, 192, 224, 256])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("heads,group", [(1, 1), (2, 3), (4, 4), (8, 2), (3, 5), (6, 8), (2, 16), (1, 33)])
@pytest.mark.parametrize("shape", [dict(new=[1, 1], ctx=[200, 90]), dict(new=[3, 2], ctx=[77, 500], tree=9),
                                   dict(new=[40, 9], ctx=[200, 90], tree=9)], ids=str)
def test_head_shapes(K, dim, dtype, heads, group, shape):
    """Every pairing of heads that a workgroup may take together, elements that fill its pieces and not."""
    p = Problem(dim=dim, dtype=dtype, heads=heads, group=group, seed=dim, **shape)
    out, lse, _ = run(K, p)
    check(p, out, lse)


@pytest.mark.parametrize("dim", [64, 96, 128, 256])
@pytest.mark.parametrize("heads,group", [(1, 5), (4, 4), (2, 8)])
@pytest.mark.parametrize("shape", [dict(new=[1, 2, 1], ctx=[5 * 512 - 3, 700, 29 * 512]),
                                   dict(new=[1, 1], ctx=[33 * 512 + 7, 41 * 512]),
                                   dict(new=[37], ctx=[3 * 1024 + 5]),
                                   dict(new=[9, 20], ctx=[37 * 1024 + 11, 900], tree=3)], ids=str)
def test_splits(K, dim, heads, group, shape):
    p = Problem(dim=dim, heads=heads, group=group, seed=dim, **shape)
    out, lse, _ = run(K, p)
    check(p, out, lse)


@pytest.mark.parametrize("requests,heads,group,dim,longest", [(511, 1, 4, 64, 1500), (512, 1, 4, 64, 1500),
                                                              (127, 8, 8, 32, 1100), (128, 8, 8, 32, 1100),
                                                              (1, 8, 4, 128, 1024), (1, 8, 4, 128, 1025)])
def test_many_requests(K, requests, heads, group, dim, longest):
    """On both sides of where every request has workgroups of its own, some of them longer than a
    workgroup's list of places, some empty."""
    g = torch.Generator().manual_seed(requests)
    ctx = torch.randint(0, longest, (requests,), generator=g).tolist()
    new = torch.randint(0, 2, (requests,), generator=g).tolist()
    ctx[0], new[0] = longest - 1, 1
    if requests > 2:
        ctx[-1], new[-1], ctx[1], new[1] = 6000, 1, 0, 1
    p = Problem(new=new, ctx=ctx, heads=heads, group=group, dim=dim, seed=requests)
    out, lse, _ = run(K, p)
    check(p, out, lse)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("new", [[1, 1, 1], [4, 2, 1], [30, 20, 9]], ids=str)
def test_rows_far_apart(K, dtype, new):
    """Rows whose sizes lie many powers of two apart: keys that decide alone, values of which the largest do
    not drown the others' bits."""
    p = Problem(new=new, ctx=[300, 41, 90], dtype=dtype, group=4, heads=4, dim=128, spread=6, values=0.05)
    out, lse, _ = run(K, p)
    check(p, out, lse)


@pytest.mark.parametrize("new", [[1, 1], [5, 3], [40, 17]], ids=str)
@pytest.mark.parametrize("kv", [0, 1])
def test_nan_groups(K, new, kv):
    """A NaN group of a value that a token sees makes those elements NaN, one of a key its whole result;
    where no token sees it, nothing."""
    p = Problem(new=new, ctx=[400, 90], heads=4, group=2, dim=128, tree=4, window=120)
    def set_nan(r, j, h, group):
        page, slot = p.slot(r, j)
        p.bytes[0, kv, page, slot, h, group] = 255
    set_nan(0, 10, 1, 2)                     # far behind the window
    set_nan(1, 80, 2, 3)                     # seen by all tokens of request 1
    last = new[0] - 1
    set_nan(0, 400 + last, 3, 0)             # the last token itself, which no other sees
    out, lse, _ = run(K, p)
    out, lse = out.double().cpu(), lse.cpu()
    nan = torch.zeros(out.shape, dtype=torch.bool)
    nan[p.starts[1]:p.starts[2], 4:6, 96:128] = True
    nan[last, 6:8, 0:32] = True
    if kv == 0:
        rows = nan.any(-1)
        assert torch.equal(torch.isnan(lse), rows)
        nan = rows[..., None].expand(out.shape)
    else:
        assert not torch.isnan(lse).any()
    assert torch.equal(torch.isnan(out), nan)
    clean = Problem(new=new, ctx=[400, 90], heads=4, group=2, dim=128, tree=4, window=120)
    want, _, size, delta = ref.attend(clean)
    u = ref.UNIT[p.dtype]
    tol = size * (2.1 * u + 4 * delta[..., None] + 2.0 ** -18) + 2.0 ** -24
    assert ((out - want).abs() <= tol)[~nan].all()


def test_nan_in_many_splits(K):
    """NaN groups in several splits and waves of one long request."""
    p = Problem(new=[1], ctx=[6000], heads=2, group=4, dim=64)
    for j, h, group in ((5, 0, 0), (700, 0, 1), (3100, 1, 0), (5999, 1, 0)):
        page, slot = p.slot(0, j)
        p.bytes[0, 1, page, slot, h, group] = 254 if j == 700 else 255
    out, lse, _ = run(K, p)
    nan = torch.isnan(out[0].cpu())
    assert nan[:4].all() and nan[4:, :32].all() and not nan[4:, 32:].any()
    assert torch.isfinite(lse).all()


@pytest.mark.parametrize("new", [[2], [50]], ids=str)
def test_infinite_queries(K, new):
    """An infinite query element gives NaN or what its sign leaves, never a result that looks like one."""
    p = Problem(new=new, ctx=[100], dtype="fp16", heads=1, group=1)
    p.q[0, 0, 3] = math.nan
    out, lse, _ = run(K, p)
    assert torch.isnan(out[0]).all() and torch.isnan(lse[0]).all()
    assert torch.isfinite(out[1:]).all() and torch.isfinite(lse[1:]).all()


def test_pages_that_are_none(K):
    """Slots of pages outside the pool are not seen; a request all of whose are gives zeros."""
    for new in ([1, 1], [6, 6], [40, 40]):
        p = Problem(new=new, ctx=[200, 20], heads=2, group=4, tree=2)
        p.table[0, 1], p.table[0, 3], p.table[1, :] = -1, p.blocks + 5, 2 ** 31 - 1
        out, lse, _ = run(K, p)
        check(p, out, lse)


def test_strides_and_no_lse(K):
    """Queries out of a fused projection, results into a wider buffer, no lse."""
    p = Problem(new=[1, 3, 9], ctx=[200, 20, 64], heads=2, group=4, dim=128)
    view, batch, scores = p.gpu(K)
    wide = torch.zeros((p.tokens, 3 * p.q_heads, p.dim), dtype=p.q.dtype, device="cuda")
    wide[:, 4:4 + p.q_heads] = p.q.cuda()
    target = torch.full((p.tokens, 2 * p.q_heads, p.dim), 5.0, dtype=p.q.dtype, device="cuda")
    ws = torch.empty(max(16, K.kvx_attend_workspace(view, batch, p.q_heads)), dtype=torch.uint8, device="cuda")
    K.kvx_attend(view, batch, scores, 0, wide[:, 4:4 + p.q_heads], target[:, p.q_heads:], None, ws)
    out, lse, _ = run(K, p)
    assert torch.equal(target[:, p.q_heads:], out) and (target[:, :p.q_heads] == 5.0).all()


def test_tokens_of_no_request(K):
    p = Problem(new=[2, 3], ctx=[20, 64])
    view, batch, scores = p.gpu(K)
    starts = torch.tensor([0, 2, 4], dtype=torch.int32).cuda()
    batch = K.make_batch(starts, batch.keep[1], 5, 3, p.max_context)
    out = torch.full((5, p.q_heads, p.dim), 5.0, dtype=p.q.dtype, device="cuda")
    ws = torch.empty(max(16, K.kvx_attend_workspace(view, batch, p.q_heads)), dtype=torch.uint8, device="cuda")
    K.kvx_attend(view, batch, scores, 0, p.q.cuda(), out, None, ws)
    assert (out[4] == 5.0).all() and torch.isfinite(out[:4]).all() and (out[:4] != 5.0).any()


@pytest.mark.parametrize("case", [dict(new=[1, 1, 1], ctx=[3000, 41, 700], heads=4, group=4, dim=128),
                                  dict(new=[9, 20, 30], ctx=[3000, 41, 700], heads=2, group=4, dim=64, tree=1)],
                         ids=str)
def test_captured(K, case):
    """Two graphs on streams of their own that share nothing but the cache, replayed with new queries and
    lengths, eager calls between."""
    p = Problem(**case)
    view, batch, scores = p.gpu(K)
    nbytes = max(16, K.kvx_attend_workspace(view, batch, p.q_heads))
    parts = []
    for _ in range(2):
        q = p.q.cuda()
        out = torch.zeros_like(q)
        lse = torch.zeros(q.shape[:2], device="cuda")
        ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.stream(stream):
            K.kvx_attend(view, batch, scores, 0, q, out, lse, ws, stream=stream)
            stream.synchronize()
            with torch.cuda.graph(graph, stream=stream):
                K.kvx_attend(view, batch, scores, 0, q, out, lse, ws, stream=stream)
        parts.append((q, out, lse, graph, stream))
    g = torch.Generator().manual_seed(1)
    for step in range(3):
        rows = [torch.randn(p.q.shape, generator=g).to(p.q.dtype) for _ in parts]
        for (q, *_), x in zip(parts, rows):
            q.copy_(x)
        torch.cuda.synchronize()
        for *_, graph, stream in parts:
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for (q, out, lse, *_), x in zip(parts, rows):
            p.q = x
            check(p, out, lse)
            eager = run(K, p, q=q)
            assert torch.equal(eager[0], out) and torch.equal(eager[1], lse)


def test_repeats_bit_for_bit(K):
    p = Problem(new=[1, 5], ctx=[9000, 1200], heads=4, group=4, dim=128)
    a, b = run(K, p), run(K, p)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_after_append_and_commit(K):
    """A step as an engine takes it: a drafted tree's rows appended, attended, its path committed, and the
    next token attends to what was moved."""
    g = torch.Generator().manual_seed(2)
    H, G, D, n, ctx = 2, 4, 128, 7, 50
    cache = torch.zeros((1, 2, 6, 16, H, D // 2), dtype=torch.uint8, device="cuda")
    scales = torch.full((1, 2, 6, 16, H, D // 32), 255, dtype=torch.uint8, device="cuda")
    table = torch.tensor([[4, 1, 5, 2]], dtype=torch.int32).cuda()
    view = K.make_cache(cache, scales, table, dtype=K.E2M1)

    def int32(v):
        return torch.tensor(v, dtype=torch.int32).cuda()

    def rope(m):
        return K.make_rope(torch.zeros(0, device="cuda"), [0], torch.zeros((1, m), dtype=torch.int32, device="cuda"))

    k, v = (torch.randn((ctx + n, H, D), generator=g).bfloat16() for _ in range(2))
    first = K.make_batch(int32([0, ctx]), int32([0]), ctx, ctx, 64)
    K.kvx_append(view, first, rope(ctx), 0, None, k[:ctx].cuda(), v[:ctx].cuda(), None)
    drafted = K.make_batch(int32([0, n]), int32([ctx]), n, n, 64)
    K.kvx_append(view, drafted, rope(n), 0, None, k[ctx:].cuda(), v[ctx:].cuda(), None)
    lens = int32([0])
    K.kvx_commit(view, 0, 1, int32([ctx]), int32([[0, 3, 6]]), int32([3]), lens)
    assert lens.tolist() == [ctx + 3]
    keep = torch.tensor(list(range(ctx)) + [ctx, ctx + 3, ctx + 6])
    kk, vv = (four.dequantise(*four.quantise(x[keep])) for x in (k, v))
    q = torch.randn((1, H * G, D), generator=g).bfloat16()
    one = K.make_batch(int32([0, 1]), int32([ctx + 2]), 1, 1, 64)
    out = torch.empty_like(q).cuda()
    ws = torch.empty(max(16, K.kvx_attend_workspace(view, one, H * G)), dtype=torch.uint8, device="cuda")
    K.kvx_attend(view, one, K.make_scores(D ** -0.5), 0, q.cuda(), out, None, ws)
    x = torch.einsum("hgd,thd->hgt", q[0].double().view(H, G, D), kk) * D ** -0.5
    w = torch.softmax(x, -1)
    want = torch.einsum("hgt,thd->hgd", w, vv).reshape(H * G, D)
    size = torch.einsum("hgt,thd->hgd", w, vv.abs()).reshape(H * G, D)
    assert ((out[0].double().cpu() - want).abs() <= size * (2.1 * 2.0 ** -8 + 1e-4) + 1e-7).all()


def test_offsets_past_32_bits(K):
    """Pages at the end of a pool whose planes hold 8.6 GB."""
    blocks, page, H, G, D = 2 ** 19, 16, 8, 4, 256
    cache = torch.zeros((1, 2, blocks, page, H, D // 2), dtype=torch.uint8, device="cuda")
    scales = torch.full((1, 2, blocks, page, H, D // 32), 255, dtype=torch.uint8, device="cuda")
    table = torch.tensor([[blocks - 1, blocks // 2 + 3, blocks - 9]], dtype=torch.int32).cuda()
    g = torch.Generator().manual_seed(6)
    code = torch.randint(0, 16, (2, 3, page, H, D), generator=g)
    byte = torch.randint(124, 128, (2, 3, page, H, D // 32), generator=g)
    at = table[0].long()
    cache[0][:, at] = four.pack(code).cuda()
    scales[0][:, at] = byte.to(torch.uint8).cuda()
    view = K.make_cache(cache, scales, table, dtype=K.E2M1)
    values = four.dequantise(code, byte).flatten(1, 2)
    for n in (1, 24):
        q = torch.randn((n, H * G, D), generator=g).bfloat16()
        batch = K.make_batch(torch.tensor([0, n], dtype=torch.int32).cuda(),
                             torch.tensor([48 - n], dtype=torch.int32).cuda(), n, n, 48)
        out = torch.empty_like(q).cuda()
        ws = torch.empty(max(16, K.kvx_attend_workspace(view, batch, H * G)), dtype=torch.uint8, device="cuda")
        K.kvx_attend(view, batch, K.make_scores(0.02), 0, q.cuda(), out, None, ws)
        x = torch.einsum("nhgd,thd->nhgt", q.double().view(n, H, G, D), values[0]) * 0.02
        seen = torch.arange(48)[None] <= 48 - n + torch.arange(n)[:, None]
        w = torch.softmax(torch.where(seen[:, None, None], x, -math.inf), -1)
        want = torch.einsum("nhgt,thd->nhgd", w, values[1]).reshape(n, H * G, D)
        size = torch.einsum("nhgt,thd->nhgd", w, values[1].abs()).reshape(n, H * G, D)
        assert ((out.double().cpu() - want).abs() <= size * (2.1 * 2.0 ** -8 + 1e-4) + 1e-7).all()
