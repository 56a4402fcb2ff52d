"""kvx_attend with up to 16 query rows per KV head: weights keep 16 bits and more in
the product with V, so that the output's own rounding is what is left."""
import pytest
import torch

import operator_reference as ref
from operator_reference import UNIT, Problem
from test_gpu_attend import TYPES, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def K():
    import paper_2509_17542_amd as K
    return K


@pytest.mark.parametrize("dim", [64, 80, 128, 256])
@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("shape", [dict(new=[1], ctx=[300], group=4), dict(new=[1, 1], ctx=[1700, 90], group=2),
                                   dict(new=[4, 3], ctx=[200, 700], group=4, tree=2),
                                   dict(new=[2], ctx=[600], softcap=30.0, slopes=True)], ids=str)
def test_one_rounding(K, shape, dtype, cache, dim):
    """A weight in two 16-bit terms is off by u^2 of itself (fp16: by 2^-25 of 2^6 where
    the second term is below the normal range), scores as elsewhere; the output is
    rounded once."""
    p = Problem(dim=dim, dtype=dtype, cache=cache, seed=dim, **shape)
    out, lse, _ = run(K, p)
    want, z, size, delta = ref.attend(p)
    u = UNIT[dtype]
    tol = want.abs() * u + size * (1.1 * u * u + 4 * delta[..., None] + 2.0 ** -17) + 2.0 ** -24
    off = (out.double().cpu() - want).abs()
    assert (off <= tol).all(), (off / tol).max()
