"""Capped scores whose cap is far above them: softcap * tanh(x / softcap) to a few
units in the last place of x, for every cap."""
import pytest
import torch

from operator_reference import UNIT, Problem
from test_gpu_attend import run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def K():
    import paper_2509_17542_amd as K
    return K


def reference(p):
    """out, lse, weights, the sum of |p v| and a bound of the scores' error, which has
    no term of the cap's size: tanh's series up to |y| = 1/4, six roundings of x's
    size; from there on an absolute error of 2^-22.2 of the cap, which is 2^-20 of x."""
    R, H, G = len(p.new), p.heads, p.q_heads // p.heads
    out = torch.zeros((p.tokens, p.q_heads, p.dim), dtype=torch.float64)
    size, lse = torch.zeros_like(out), torch.zeros((p.tokens, p.q_heads), dtype=torch.float64)
    delta = torch.zeros_like(lse)
    w = torch.zeros((R, H, p.max_context), dtype=torch.float64)
    err = torch.zeros_like(w)
    for r, n in enumerate(p.new):
        k, v = p.rows(0, r)[0], p.rows(1, r)[0]
        for i in range(n):
            tok = p.starts[r] + i
            see, distance = p.sees(r, i)
            idx = torch.nonzero(see)[:, 0]
            q = p.q[tok].double().view(H, G, p.dim)
            kk, vv = k[idx].permute(1, 2, 0), v[idx].permute(1, 0, 2)
            x = torch.matmul(q, kk) * p.scale
            d = torch.matmul(q.abs(), kk.abs()) * p.scale * (p.dim + 8) * 2.0 ** -24 + x.abs() * 2.0 ** -19.5
            x = p.softcap * torch.tanh(x / p.softcap)
            if p.slopes is not None:
                x = x - p.slopes.double().view(H, G, 1) * distance[idx].abs().double()
                d = d + x.abs() * 2.0 ** -22
            d = d + x.abs() * 2.0 ** -22 + 2.0 ** -22
            z = torch.logsumexp(x, -1)
            e = torch.exp(x - z[..., None])
            out[tok] = torch.matmul(e, vv).reshape(p.q_heads, p.dim)
            size[tok] = torch.matmul(e, vv.abs()).reshape(p.q_heads, p.dim)
            lse[tok], delta[tok] = z.reshape(-1), d.amax(-1).reshape(-1)
            # the lse that the weights' call is given is rounded to 32 bits
            e32 = torch.exp(x - z.float().double()[..., None])
            w[r][:, idx] += e32.sum(1)
            err[r][:, idx] += (2 * (d + z.abs()[..., None] * 2.0 ** -22) * e32).sum(1)
    return out, lse, size, delta, w, err + w * 2.0 ** -20 + 1e-30


CASES = {
    "few": dict(new=[1, 3], ctx=[300, 41]),
    "few_split": dict(new=[2], ctx=[900], group=4),
    "rows": dict(new=[40], ctx=[100]),
    "rows_bias": dict(new=[60], ctx=[100], slopes=True),
    "tree": dict(new=[20, 40], ctx=[90, 30], tree=3, slopes=True, dim=128),
}


@pytest.mark.parametrize("softcap", [1e-3, 30.0, 64.0, 65.0, 200.0, 1e3, 1e4, 1e6, 1e20, 3e38])
@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("fp16", "e4m3fn")])
@pytest.mark.parametrize("name", CASES)
def test_caps(K, name, dtype, cache, softcap):
    p = Problem(dtype=dtype, cache=cache, softcap=softcap, values=3.0, **CASES[name])
    out, lse, (view, batch, scores, _) = run(K, p)
    want, z, size, delta, weights, err = reference(p)
    if softcap <= 64.0:
        # caps of this size: an absolute error of 2^-21 of the cap, 3e-5 at most
        delta, err = delta + softcap * 2.0 ** -21, err + weights * 2 * softcap * 2.0 ** -21
    out, lse = out.double().cpu(), lse.double().cpu()
    tol = size * (2.1 * UNIT[dtype] + 4 * delta[..., None] + 2.0 ** -18) + 2.0 ** -24
    assert ((out - want).abs() <= tol).all(), ((out - want).abs() / tol).max()
    bad = (lse - z).abs() / (delta + 2.0 ** -21 * (1 + z.abs()))
    assert bad.max() <= 1, bad.max()
    w = torch.zeros((len(p.new), p.heads, p.max_context), device="cuda")
    K.kvx_weigh(view, batch, scores, 0, p.q.cuda(), z.float().cuda(), w)
    off = (w.double().cpu() - weights).abs()
    assert (off <= err).all(), (off / err).max()


def test_large_scores(K):
    """Scores of hundreds under caps of their size and above."""
    for softcap in (100.0, 1000.0, 1e5):
        for new in ([1], [40]):
            p = Problem(new=new, ctx=[200], softcap=softcap, values=12.0)
            out, lse, _ = run(K, p)
            want, z, size, delta, _, _ = reference(p)
            tol = size * (2.1 * UNIT["bf16"] + 4 * delta[..., None] + 2.0 ** -18) + 2.0 ** -24
            assert ((out.double().cpu() - want).abs() <= tol).all()
            assert ((lse.double().cpu() - z).abs() <= delta + 2.0 ** -21 * (1 + z.abs())).all()


def test_smallest_caps(K):
    """All scores next to 0, an exact 0 too: every slot weighs the same."""
    for new in ([1], [40]):
        p = Problem(new=new, ctx=[100], softcap=1e-40)
        p.q[0] = 0
        out, lse, _ = run(K, p)
        want, z, size, _, _, _ = reference(p)
        assert ((out.double().cpu() - want).abs() <= size * (2.1 * UNIT["bf16"] + 2.0 ** -18) + 2.0 ** -24).all()
        assert ((lse.double().cpu() - z).abs() <= 2.0 ** -21 * (1 + z.abs())).all()
