"""Values that are not finite, in slots that a token sees: infinite results whatever
the slot's weight, NaN where infinities oppose; the other elements, and the tokens
that do not see the slot, are as if it were not there.  The same wherever the slot
lies: in a tile that all rows see whole or in part, in any split."""
import math

import pytest
import torch

import operator_reference as ref
from operator_reference import UNIT, Problem
from test_gpu_attend import TYPES, run

pytestmark = pytest.mark.gpu

SHAPES = {
    "few": dict(new=[1], ctx=[300]),
    "few_tree": dict(new=[3], ctx=[200], tree=3),
    "few_32": dict(new=[8], ctx=[500], group=4),
    "few_split": dict(new=[1, 2], ctx=[1300, 600], group=4),
    "few_many_splits": dict(new=[1], ctx=[33 * 512 + 9], heads=1),
    "rows_64": dict(new=[20], ctx=[200], group=3, dim=128),
    "rows": dict(new=[70], ctx=[300]),
    "rows_tree": dict(new=[70], ctx=[300], tree=5),
    "rows_split": dict(new=[40], ctx=[700]),
    "wide_heads": dict(new=[1, 20], ctx=[300, 100], dim=192),
}


@pytest.fixture(scope="module")
def K():
    import paper_2509_17542_amd as K
    return K


def check(p, out):
    want, _, size, delta = ref.attend(p)
    out = out.double().cpu()
    assert not torch.isfinite(want).all()
    assert torch.equal(torch.isnan(out), torch.isnan(want))
    endless = torch.isinf(want)
    assert torch.equal(torch.isinf(out), endless) and torch.equal(out[endless], want[endless])
    tol = size * (2.1 * UNIT[p.dtype] + 4 * delta[..., None] + 2.0 ** -18) + 2.0 ** -24
    assert ((out - want).abs() <= tol)[torch.isfinite(want)].all()


def put(p, r, j, head, at, value):
    """Element `at` of V's row becomes infinite or NaN."""
    page, slot = p.slot(r, j)
    if p.kind == "e4m3fn":                       # has no infinity: the row's scale does, or its code is NaN
        if math.isnan(value):
            p.cache.view(torch.uint8)[p.layer, 1, page, slot, head, at] = 0x7F
        else:
            p.scales[p.layer, 1, page, slot, head] = value
    elif p.kind == "e5m2":
        code = 0x7F if math.isnan(value) else 0x7C if value > 0 else 0xFC
        p.cache.view(torch.uint8)[p.layer, 1, page, slot, head, at] = code
    else:
        p.cache[p.layer, 1, page, slot, head, at] = value


@pytest.mark.parametrize("hole", [False, True], ids=["whole", "part"])
@pytest.mark.parametrize("steep", [0.0, 40.0, 400.0])
@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("name", SHAPES)
def test_seen(K, name, dtype, cache, steep, hole):
    """steep: the bias by distance that the first slots have, so that their weights are
    zero in 16 bits (40) or in 32 (400).  A hole (a page that is none) near the slots
    makes their tile one that no row sees whole."""
    p = Problem(dtype=dtype, cache=cache, **SHAPES[name])
    if steep:
        p.slopes = torch.full((p.q_heads,), steep / p.max_context)
    if hole:
        p.table[:, 1] = -1
    # a hole hides slots 16 to 31
    for r, c in enumerate(p.ctx):
        put(p, r, 3, 0, 3, math.inf)
        put(p, r, 5, 0, 7, -math.inf)
        put(p, r, 40, p.heads - 1, 9, math.nan)
        put(p, r, 7, p.heads - 1, 11, math.inf)
        if c > 70:
            put(p, r, 70, p.heads - 1, 11, -math.inf)
    out, _, _ = run(K, p)
    check(p, out)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("name", ["few", "rows", "rows_split"])
def test_infinite_codes_with_odd_scales(K, name, dtype):
    """An infinite code times a zero scale is NaN, times a negative one the other
    infinity; an infinite or NaN scale makes infinities or NaN of the row."""
    p = Problem(dtype=dtype, cache="e5m2", **SHAPES[name])
    for j, scale in ((33, 0.0), (34, -1.0), (90, math.inf), (120, math.nan)):
        page, slot = p.slot(0, j)
        head = int(j > 60)
        p.scales[p.layer, 1, page, slot, head] = scale
        if head == 0:
            p.cache.view(torch.uint8)[p.layer, 1, page, slot, head, j % 8] = 0x7C
    if name != "few":
        p.scales[p.layer, 1, p.slot(0, 120)[0], p.slot(0, 120)[1], 1] = 1.0   # infinities alone
        page, slot = p.slot(0, 90)
        p.cache.view(torch.uint8)[p.layer, 1, page, slot, 1, 5] = 0           # 0 times infinity
    out, _, _ = run(K, p)
    check(p, out)


def test_one_split_alone_holds_it(K):
    """The split with the infinity weighs nothing beside the others."""
    for new, ctx in ([1], 3 * 512 + 40), ([1], 40 * 512), ([40], 900):
        p = Problem(new=new, ctx=[ctx], dtype="fp16", cache="fp16")
        p.slopes = torch.full((p.q_heads,), 600.0 / ctx)
        put(p, 0, 2, 1, 4, -math.inf)
        out, _, _ = run(K, p)
        check(p, out)
