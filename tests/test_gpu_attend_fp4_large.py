"""kvx_attend over a 4-bit cache whose planes hold 2^32 groups, which the few-rows kernel does
not number: calls of few rows keep the precision that they have over other pools."""
import math

import pytest
import torch

import operator_reference as ref
from operator_reference import UNIT
from test_gpu_attend_fp4 import Problem

pytestmark = pytest.mark.gpu
GROUPS = 1 << 32          # a pool has as many, to whole pages
ROOM = GROUPS + (1 << 20)


@pytest.fixture(scope="module")
def K():
    import paper_2509_17542_amd as K
    return K


@pytest.fixture(scope="module")
def pool():
    """Codes and scale bytes of two planes, 146 GB that nobody fills."""
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 160e9:
        pytest.skip("needs 146 GB of device memory")
    codes = torch.empty(2 * ROOM * 16, dtype=torch.uint8, device="cuda")
    scales = torch.empty(2 * ROOM, dtype=torch.uint8, device="cuda")
    yield codes, scales
    del codes, scales
    torch.cuda.empty_cache()


def place(K, p, pool):
    """The problem's pages at the pool's end, middle and beginning: the view of it."""
    blocks = -(-GROUPS // (p.page * p.heads * p.dim // 32))
    shape = (1, 2, blocks, p.page, p.heads)
    codes, scales = (x[:math.prod(shape) * n].view(*shape, n) for x, n in zip(pool, (p.dim // 2, p.dim // 32)))
    table = p.table.clone()
    for i, old in enumerate(sorted(set(p.table[p.table >= 0].tolist()))):
        new = (blocks - 1 - i, blocks // 2 + i, i)[i % 3]
        table[p.table == old] = new
        for kv in range(2):
            codes[0, kv, new].copy_(p.codes[0, kv, old])
            scales[0, kv, new].copy_(p.bytes[0, kv, old])
    return K.make_cache(codes, scales, table.cuda(), dtype=K.E2M1)


def one_rounding(p, out, lse):
    """Weights in two bf16 terms are off by 2^-16 of themselves, a tenth for the other roundings, the scores
    as elsewhere; the output is rounded once."""
    want, z, size, delta = ref.attend(p)
    tol = want.abs() * UNIT[p.dtype] + size * (1.1 * 2.0 ** -16 + 4 * delta[..., None] + 2.0 ** -17) + 2.0 ** -24
    off = (out.double().cpu() - want).abs()
    assert (off <= tol).all(), (off / tol).max()
    assert ((lse.double().cpu() - z).abs() <= delta + 2.0 ** -21 * (1 + z.abs())).all()


def attend(K, p, view, batch, scores):
    q = p.q.cuda()
    out, lse = torch.full_like(q, math.nan), torch.full(q.shape[:2], math.nan, device="cuda")
    ws = torch.full((max(16, K.kvx_attend_workspace(view, batch, p.q_heads)),), 0xFF, dtype=torch.uint8, device="cuda")
    K.kvx_attend(view, batch, scores, 0, q, out, lse, ws)
    return out, lse


SHAPES = [dict(new=[1], ctx=[300], heads=4, group=4, dim=128), dict(new=[1, 1], ctx=[1700, 90], heads=2, group=2, dim=64),
          dict(new=[4, 3], ctx=[200, 700], heads=2, group=4, dim=256, tree=2),
          dict(new=[2], ctx=[600], heads=1, group=8, dim=96, softcap=30.0, slopes=True),
          dict(new=[1], ctx=[5000], heads=8, group=2, dim=128, window=3000),
          dict(new=[1, 1], ctx=[900, 12], heads=2, group=16, dim=32, softcap=100.0)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_one_rounding(K, shape, dtype):
    """Over a pool of the usual size."""
    p = Problem(dtype=dtype, seed=shape["dim"], **shape)
    view, batch, scores = p.gpu(K)
    one_rounding(p, *attend(K, p, view, batch, scores))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_one_rounding_of_large_pools(K, pool, shape, dtype):
    p = Problem(dtype=dtype, seed=shape["dim"], **shape)
    _, batch, scores = p.gpu(K)
    one_rounding(p, *attend(K, p, place(K, p, pool), batch, scores))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_more_rows_and_rows_read_back(K, pool, dtype):
    """What the many-rows kernel takes in any case, and kvx_fetch, over such a pool."""
    p = Problem(dtype=dtype, new=[40, 9], ctx=[200, 700], heads=2, group=4, dim=128, tree=2)
    view, batch, scores = place(K, p, pool), *p.gpu(K)[1:]
    out, lse = attend(K, p, view, batch, scores)
    want, _, size, delta = ref.attend(p)
    off = (out.double().cpu() - want).abs()
    assert (off <= size * (2.1 * UNIT[dtype] + 4 * delta[..., None] + 2.0 ** -18) + 2.0 ** -24).all()
    k, v = (torch.empty((p.tokens, p.heads, p.dim), dtype=p.q.dtype, device="cuda") for _ in range(2))
    K.kvx_fetch(view, batch, 0, k, v)
    for kv, got in enumerate((k, v)):
        rows = torch.cat([p.rows(kv, r)[0][c:c + n] for r, (n, c) in enumerate(zip(p.new, p.ctx))])
        assert torch.equal(got.cpu(), rows.to(p.q.dtype))
