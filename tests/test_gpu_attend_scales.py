"""kvx_attend over 8-bit rows whose scales differ widely: those of slots that a
token does not see have no part in its result, and small rows beside large ones
keep their bits."""
import pytest
import torch

import operator_reference as ref
from operator_reference import FLOAT8, FMAX, UNIT, Problem
from test_gpu_attend import run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def K():
    import paper_2509_17542_amd as K
    return K


def check(p, out, lse, keep):
    """The tolerance of ordinary rows, and a weight's rounding below the normal
    range: its product with the row's scale is held to 2^-25 where the row's largest
    is 2^10 or more, and that largest, times the largest code, is one of the terms of
    `size` (every row has a code that large)."""
    want, z, size, delta = ref.attend(p)
    out, lse = out.double().cpu(), lse.double().cpu()
    small = size.amax(-1, keepdim=True) * max(p.total) * 2.0 ** -35
    tol = size * (2.1 * UNIT[p.dtype] + 4 * delta[..., None] + 2.0 ** -18) + small + 2.0 ** -24
    assert torch.isfinite(out[keep]).all()
    assert ((out - want).abs() <= tol)[keep].all(), ((out - want).abs() / tol)[keep].max()
    assert ((lse - z).abs() <= delta + 2.0 ** -21 * (1 + z.abs()))[keep].all()


UNSEEN = {
    "tree": dict(new=[3], ctx=[40], tree=3),
    "trees": dict(new=[20, 30], ctx=[40, 0], tree=7),
    "tree_wide": dict(new=[90], ctx=[40], tree=8, group=4),
    "chain": dict(new=[4, 2], ctx=[600, 61]),
    "chain_wide": dict(new=[60], ctx=[300]),
    "window": dict(new=[1, 9], ctx=[77, 205], window=33),
    "window_wide": dict(new=[70], ctx=[300], window=33, prefix=[5]),
    "window_split": dict(new=[1], ctx=[1300], window=700),
}


@pytest.mark.parametrize("scale", [1e30, 2.0 ** 16, 2.0 ** 4])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("cache", ["e4m3fn", "e5m2"])
@pytest.mark.parametrize("name", UNSEEN)
def test_not_seen(K, name, cache, dtype, scale):
    """Large scales (and keys' scales) where no token sees them, and in every
    request's last token, which is left out with those that see it."""
    p = Problem(dtype=dtype, cache=cache, **UNSEEN[name])
    keep, spoilt = [], 0
    for r, n in enumerate(p.new):
        sees = torch.stack([p.sees(r, i)[0] for i in range(n)])
        which = ~sees.any(0)
        if n > 1:
            which[p.total[r] - 1] = True
        for j in torch.nonzero(which)[:, 0].tolist():
            page, slot = p.slot(r, j)
            p.scales[p.layer, :, page, slot] = scale
            spoilt += 1
        keep += [p.starts[r] + i for i in range(n) if not (sees[i] & which).any()]
    assert spoilt and keep
    out, lse, _ = run(K, p)
    check(p, out, lse, keep)


SEEN = {
    "few": dict(new=[1, 2], ctx=[300, 41]),
    "few_32": dict(new=[8], ctx=[600], group=4),
    "few_split": dict(new=[1], ctx=[1300], group=4),
    "rows": dict(new=[40], ctx=[200]),
    "rows_split": dict(new=[100], ctx=[700]),
    "tree": dict(new=[50], ctx=[100], tree=2),
}


@pytest.mark.parametrize("small", [1.0, 2.0 ** -10])
@pytest.mark.parametrize("slopes", [0.0, 0.25])
@pytest.mark.parametrize("cache", ["e4m3fn", "e5m2"])
@pytest.mark.parametrize("name", SEEN)
def test_seen(K, name, cache, slopes, small):
    """Rows with an element of 60000 among rows of ordinary and of small size; with a
    bias by distance the large ones weigh next to nothing."""
    p = Problem(dtype="fp16", cache=cache, values=2.0, **SEEN[name])
    if slopes:
        p.slopes = torch.full((p.q_heads,), slopes)
    p.scales[:, 1] *= small
    g = torch.Generator().manual_seed(1)
    bits = p.cache.view(torch.uint8)
    s = 60000.0 / FMAX[cache]
    for r, t in enumerate(p.total):
        for j in {0, 9, t // 3, t // 2}:
            page, slot = p.slot(r, j)
            row = torch.randn((p.heads, p.dim), generator=g) * small
            row[:, j % p.dim] = 60000.0 if j % 2 else -60000.0
            bits[p.layer, 1, page, slot] = (row / s).to(FLOAT8[cache]).view(torch.uint8)
            p.scales[p.layer, 1, page, slot] = s
    out, lse, _ = run(K, p)
    check(p, out, lse, range(p.tokens))


@pytest.mark.parametrize("cache", ["e4m3fn", "e5m2"])
@pytest.mark.parametrize("shape", [dict(new=[1], ctx=[1500]), dict(new=[40], ctx=[400])], ids=str)
def test_scores_that_grow(K, shape, cache):
    """Weights that rise by orders of magnitude along the slots, scales that fall: what
    was large at first is not in the end."""
    p = Problem(dtype="fp16", cache=cache, **shape)
    p.slopes = torch.full((p.q_heads,), 60.0 / p.max_context)
    t = p.total[0]
    for j in range(t):
        page, slot = p.slot(0, j)
        p.scales[p.layer, 1, page, slot] *= 2.0 ** (12.0 - 24.0 * j / t)
    out, lse, _ = run(K, p)
    check(p, out, lse, range(p.tokens))
