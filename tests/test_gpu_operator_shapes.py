"""Forms of the decode operators by the size of a head, the query rows of a KV head,
the scores and the place in a large cache, each against the plain form in 64 bits."""

import pytest
import torch

import operator_reference as ref
from operator_reference import UNIT, Problem
from test_gpu_attend import TYPES, check, run

pytestmark = pytest.mark.gpu

SCORES = {"plain": {}, "bias": dict(slopes=True), "capped": dict(softcap=20.0, values=2.0),
          "both": dict(softcap=30.0, slopes=True, window=70)}


@pytest.fixture(scope="module")
def K():
    import paper_2509_17542_amd as K
    return K


def weigh(K, p):
    view, batch, scores = p.gpu(K)
    lse = ref.attend(p)[1].float()
    start = torch.rand((len(p.new), p.heads, p.max_context + 3))
    w = start.cuda()
    K.kvx_weigh(view, batch, scores, p.layer, p.q.cuda(), lse.cuda(), w)
    want, tol = ref.weigh(p, lse, start)
    got = w.double().cpu()
    assert ((got - want).abs() <= tol).all(), (got - want).abs().max()
    for r, t in enumerate(p.total):
        assert torch.equal(w[r, :, t:].cpu(), start[r, :, t:])


@pytest.mark.parametrize("shape", [dict(new=[1, 2], ctx=[200, 61], group=3), dict(new=[20, 9], ctx=[200, 61], tree=4)],
                         ids=["few", "many"])
@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("dim", [16, 80, 96, 112, 128, 144, 192, 256])
def test_weigh_head_dims(K, dim, dtype, cache, shape):
    weigh(K, Problem(dim=dim, dtype=dtype, cache=cache, seed=dim, **shape))


@pytest.mark.parametrize("shape", [dict(new=[1, 2], ctx=[200, 61], group=3), dict(new=[20, 9], ctx=[200, 61], tree=4)],
                         ids=["few", "many"])
@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("fp16", "e4m3fn")])
@pytest.mark.parametrize("scores", ["bias", "capped", "both"])
@pytest.mark.parametrize("dim", [80, 128, 192, 256])
def test_weigh_scores(K, dim, scores, dtype, cache, shape):
    weigh(K, Problem(dim=dim, dtype=dtype, cache=cache, seed=dim, **shape, **SCORES[scores]))


@pytest.mark.parametrize("scores", SCORES)
@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("dim", [64, 80, 112, 128])
def test_17_to_32_rows(K, dim, dtype, cache, scores):
    p = Problem(new=[6, 8, 1], ctx=[700, 41, 64], group=4, tree=3, dim=dim, dtype=dtype, cache=cache, seed=dim,
                **SCORES[scores])
    out, lse, _ = run(K, p)
    check(p, out, lse)


@pytest.mark.parametrize("shape", [dict(new=[1, 2], ctx=[200, 61], group=3), dict(new=[30, 9], ctx=[200, 61], tree=4),
                                   dict(new=[90], ctx=[300])], ids=["few", "rows_64", "rows"])
@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "e4m3fn"), ("fp16", "e5m2")])
@pytest.mark.parametrize("scores", ["bias", "capped", "both"])
@pytest.mark.parametrize("dim", [80, 128, 192, 256])
def test_attend_scores(K, dim, scores, dtype, cache, shape):
    p = Problem(dim=dim, dtype=dtype, cache=cache, seed=dim, **shape, **SCORES[scores])
    out, lse, _ = run(K, p)
    check(p, out, lse)


# ---- pages past 2^32 elements of a plane --------------------------------------

PAGE, HEADS, DIM = 64, 8, 128
LOW = 64                                         # pages that such places fall on when cut to 32 bits
BLOCKS = (1 << 32) // (PAGE * HEADS * DIM) + LOW


@pytest.fixture
def large():
    x = torch.empty((1, 2, BLOCKS, PAGE, HEADS, DIM), dtype=torch.bfloat16, device="cuda")
    x[:, :, :LOW] = 7.0
    yield x
    del x
    torch.cuda.empty_cache()


def moved(K, large, **shape):
    """A problem whose pages are the large cache's last ones, and its view."""
    p = Problem(heads=HEADS, dim=DIM, page=PAGE, **shape)
    table = p.table.clone()
    for n, b in enumerate(sorted(set(p.table[p.table >= 0].tolist()))):
        assert n < LOW
        large[0, :, BLOCKS - 1 - n] = p.cache[0, :, b].cuda()
        table[p.table == b] = BLOCKS - 1 - n
    _, batch, scores = p.gpu(K)
    return p, K.make_cache(large, None, table.cuda()), batch, scores, table


def row(large, table, r, j):
    return large[0, :, int(table[r, j // PAGE]), j % PAGE]


def test_weigh_past_32_bits(K, large):
    p, view, batch, scores, _ = moved(K, large, new=[1, 20], ctx=[100, 300], group=2)
    lse = ref.attend(p)[1].float()
    w = torch.zeros((2, HEADS, p.max_context), device="cuda")
    K.kvx_weigh(view, batch, scores, 0, p.q.cuda(), lse.cuda(), w)
    want, tol = ref.weigh(p, lse, torch.zeros(w.shape))
    assert ((w.double().cpu() - want).abs() <= tol).all()


def test_append_past_32_bits(K, large):
    p, view, batch, _, table = moved(K, large, new=[3, 20], ctx=[100, 300], group=2)
    k, v = (torch.randn((p.tokens, HEADS, DIM)).bfloat16() for _ in range(2))
    inv_freq = 10000.0 ** (-torch.arange(DIM // 2, dtype=torch.float32) / (DIM // 2))
    positions = torch.arange(p.tokens, dtype=torch.int32)[None]
    rope = K.make_rope(inv_freq.cuda(), [DIM // 2], positions.cuda())
    K.kvx_append(view, batch, rope, 0, None, k.cuda(), v.cuda(), None)
    turned = ref.rotate(k, inv_freq, [DIM // 2], positions, False)
    for r, n in enumerate(p.new):
        for i in range(n):
            got = row(large, table, r, p.ctx[r] + i).double().cpu()
            want = turned[p.starts[r] + i]
            slack = want.abs().amax(-1, keepdim=True) * 2.0 ** -20 + 2.0 ** -25
            assert ((got[0] - want).abs() <= want.abs() * UNIT["bf16"] + slack).all()
            assert torch.equal(got[1], v[p.starts[r] + i].double())
    assert (large[:, :, :LOW] == 7.0).all()


def test_evict_past_32_bits(K, large):
    p, view, _, _, table = moved(K, large, new=[0, 0], ctx=[900, 100])
    w = torch.rand((1, 2, HEADS, 900))
    before = [torch.stack([row(large, table, r, j).cpu() for j in range(t)]) for r, t in enumerate(p.ctx)]
    d = w.cuda()
    kept = torch.zeros((1, 2, HEADS, 300), dtype=torch.int32, device="cuda")
    new_lens = torch.zeros(2, dtype=torch.int32, device="cuda")
    K.kvx_evict(view, 0, 1, torch.tensor(p.ctx, dtype=torch.int32).cuda(), 900, 300, 4, 40, d, d, kept, new_lens)
    assert new_lens.tolist() == [300, 100]
    for r, t in enumerate(p.ctx):
        after = torch.stack([row(large, table, r, j).cpu() for j in range(t)])
        for h in range(HEADS):
            stay = ref.evict(t, 300, 4, 40, w[0, r, h].tolist())
            assert torch.equal(after[:len(stay), :, h].view(torch.int16), before[r][stay][:, :, h].view(torch.int16))
    assert (large[:, :, :LOW] == 7.0).all()


def test_commit_past_32_bits(K, large):
    p, view, _, _, table = moved(K, large, new=[30, 64], ctx=[100, 41])
    before = [torch.stack([row(large, table, r, j).cpu() for j in range(t)]) for r, t in enumerate(p.total)]
    paths = [[1, 5, 6, 29], [0, 1, 40, 63]]
    ints = lambda x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    new_lens = torch.zeros(2, dtype=torch.int32, device="cuda")
    K.kvx_commit(view, 0, 1, ints(p.ctx), ints(paths), ints([4, 4]), new_lens)
    assert new_lens.tolist() == [104, 45]
    for r, path in enumerate(paths):
        c = p.ctx[r]
        after = torch.stack([row(large, table, r, j).cpu() for j in range(c + 4)])
        want = torch.cat([before[r][:c], before[r][[c + j for j in path]]])
        assert torch.equal(after.view(torch.int16), want.view(torch.int16))
    assert (large[:, :, :LOW] == 7.0).all()
