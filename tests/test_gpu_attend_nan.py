"""A NaN that a token sees, in its query or in a key, gives that token's heads NaN
(result, lse and weights) and no others, wherever the slot lies: alone in a wave's
share of the slots, alone in a split, or among others."""
import math

import pytest
import torch

import operator_reference as ref
from operator_reference import Problem
from test_gpu_attend import TYPES, UNIT, run

pytestmark = pytest.mark.gpu

CUTS = {
    "few": dict(new=[1, 2], ctx=[37, 90]),
    "few_32": dict(new=[8], ctx=[600], group=4, heads=2),
    "few_split": dict(new=[1, 3], ctx=[1300, 512], group=4),
    "few_many_splits": dict(new=[1], ctx=[33 * 512 + 7], group=5),
    "rows_64": dict(new=[25], ctx=[90]),
    "rows": dict(new=[70], ctx=[90]),
    "rows_split": dict(new=[40], ctx=[700]),
    "rows_many_splits": dict(new=[40], ctx=[9000]),
}


@pytest.fixture(scope="module")
def K():
    import paper_2509_17542_amd as K
    return K


def spoil(p, kv, r, j, head):
    """A NaN in one row: an element, or an 8-bit row's code or scale."""
    page, slot = p.slot(r, j)
    if p.scales is None:
        p.cache[p.layer, kv, page, slot, head, 3] = math.nan
    elif j % 2:
        p.cache.view(torch.uint8)[p.layer, kv, page, slot, head, 3] = 0x7F
    else:
        p.scales[p.layer, kv, page, slot, head] = math.nan


def check(p, out, lse):
    """As for finite values, for the rows that see no NaN; the others are NaN."""
    want, z, size, delta = ref.attend(p)
    out, lse = out.double().cpu(), lse.double().cpu()
    lost = torch.isnan(z)
    assert lost.any() and not lost.all()
    assert torch.equal(torch.isnan(lse), lost)
    assert torch.isnan(out[lost]).all()
    u = UNIT[p.dtype]
    tol = size * (2.1 * u + 4 * delta[..., None] + 2.0 ** -18) + 2.0 ** -24
    assert ((out - want).abs() <= tol)[~lost].all()
    assert ((lse - z).abs() <= delta + 2.0 ** -21 * (1 + z.abs()))[~lost].all()


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("name", CUTS)
def test_a_query(K, name, dtype, cache):
    p = Problem(dtype=dtype, cache=cache, **CUTS[name])
    p.q[0, 1, 5] = math.nan
    p.q[p.tokens - 1, p.q_heads - 1, 0] = math.nan
    out, lse, _ = run(K, p)
    check(p, out, lse)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("shape,slot", [
    (dict(new=[1], ctx=[0]), 0),                          # the only slot
    (dict(new=[1], ctx=[32]), 32),                        # alone in its wave's share
    (dict(new=[1], ctx=[300]), 70),                       # among others
    (dict(new=[1], ctx=[512], group=3), 512),             # alone in a split
    (dict(new=[1], ctx=[33 * 512]), 33 * 512),            # the same, of many
    (dict(new=[5, 2], ctx=[508, 100], group=4), 512),
    (dict(new=[40], ctx=[90]), 129),
    (dict(new=[40], ctx=[217]), 256),                     # alone in a split, seen by the last token
    (dict(new=[20], ctx=[237], group=3), 256),
    (dict(new=[40], ctx=[700]), 300),
], ids=str)
def test_a_key(K, shape, slot, dtype, cache):
    p = Problem(dtype=dtype, cache=cache, **shape)
    spoil(p, 0, 0, slot, 0)
    out, lse, _ = run(K, p)
    check(p, out, lse)


@pytest.mark.parametrize("cut", ["few", "few_split", "rows", "rows_split"])
def test_weights(K, cut):
    """The lse of such a token is passed on to the weights of what it saw."""
    p = Problem(**CUTS[cut])
    p.q[1, 0, 7] = math.nan
    _, lse, (view, batch, scores, _) = run(K, p)
    start = torch.rand((len(p.new), p.heads, p.max_context))
    w = start.cuda()
    K.kvx_weigh(view, batch, scores, 0, p.q.cuda(), lse, w)
    want, tol = ref.weigh(p, lse.cpu(), start)
    got = w.double().cpu()
    lost = torch.isnan(want)
    assert lost.any() and not lost.all()
    assert torch.equal(torch.isnan(got), lost)
    assert ((got - want).abs() <= tol)[~lost].all()
