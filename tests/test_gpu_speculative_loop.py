"""The loop of examples/decode_loop.py over a cache of 4 bits: appended, attended, verified and
committed step by step, its lengths, paths and rows stay what the operators' definitions
say; and over both caches the accepted tokens are those of the tree."""
import importlib.util
import os

import pytest
import torch

import serving_reference as four
from conftest import ROOT

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def loop():
    spec = importlib.util.spec_from_file_location("decode_loop", os.path.join(ROOT, "examples", "decode_loop.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def stored(engine, loop, layer, kv, r):
    """The rows as the cache's bytes stand for, float64."""
    at = torch.arange(engine.lens[r], device="cuda")
    page, slot = engine.table[r].long()[at // loop.PAGE], at % loop.PAGE
    return four.dequantise(four.unpack(engine.cache[layer, kv][page, slot].cpu()),
                           engine.scale_bytes[layer, kv][page, slot].cpu())


def test_four_bit_loop(loop):
    engine = loop.main(steps=12, four=True)
    assert all(n >= p + 12 for n, p in zip(engine.lens, [40, 57, 90]))
    assert engine.placed == engine.lens
    assert all(0 <= t < loop.VOCAB for t in engine.last)
    for r in range(engine.requests):
        for layer in range(loop.LAYERS):
            for kv, x in enumerate(engine.rows(r, layer)):
                want = stored(engine, loop, layer, kv, r)
                assert torch.isfinite(want).all()
                assert torch.equal(x.double().cpu(), want)


@pytest.mark.parametrize("bits", [4, 16])
def test_next_token_attends_to_what_was_accepted(loop, bits):
    """After some steps a further token's attention is that over the rows that kvx_fetch reads back."""
    engine = loop.Engine([40, 57, 90], pages=24, seed=5, four=bits == 4)
    for _ in range(5):
        engine.step(8)
    K, n = loop.K, engine.requests
    q = engine.normal(n, loop.Q_HEADS, loop.DIM).bfloat16()
    batch = K.make_batch(loop.int32(range(n + 1)), loop.int32([t - 1 for t in engine.lens]), n, 1, max(engine.lens))
    out = torch.empty_like(q)
    ws = torch.empty(max(16, K.kvx_attend_workspace(engine.view, batch, loop.Q_HEADS)), dtype=torch.uint8, device="cuda")
    K.kvx_attend(engine.view, batch, engine.scores, 1, q, out, None, ws)
    for r in range(n):
        k, v = (x.double().repeat_interleave(loop.GROUP, 1).permute(1, 0, 2).contiguous() for x in engine.rows(r, 1))
        p = torch.softmax((k @ q[r].double()[:, :, None])[..., 0] * loop.DIM ** -0.5, -1)
        want, size = (p[:, None] @ v)[:, 0], (p[:, None] @ v.abs())[:, 0]
        # two roundings to bf16 (weights, output), scores to 1e-5
        assert ((out[r].double() - want).abs() <= size * (2.1 * 2.0 ** -8 + 1e-4) + 1e-7).all()


def test_sixteen_bit_loop_grows(loop):
    """Every step accepts the token sampled last at least."""
    engine = loop.Engine([30, 41], pages=20, seed=9)
    for _ in range(6):
        before = list(engine.lens)
        engine.step(8)
        assert all(a < b <= a + 8 for a, b in zip(before, engine.lens))
