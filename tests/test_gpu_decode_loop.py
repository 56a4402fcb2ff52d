"""The decode loop of examples/decode_loop.py: lengths, weights and what attention
sees stay those of the operators' definitions over many steps."""
import importlib.util
import os

import pytest
import torch

from conftest import ROOT

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def loop():
    spec = importlib.util.spec_from_file_location("decode_loop", os.path.join(ROOT, "examples", "decode_loop.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def rows_of(engine, loop, layer, kv, r):
    at = torch.arange(engine.lens[r], device="cuda")
    return engine.cache[layer, kv, engine.table[r].long()[at // loop.PAGE], at % loop.PAGE]


def test_loop(loop):
    engine = loop.main(steps=12)
    assert all(n <= loop.BUDGET + loop.PAGE + 8 for n in engine.lens)
    assert all(p >= n for p, n in zip(engine.placed, engine.lens))
    # one more token of each request against plain attention over the slots in use
    K, n = loop.K, engine.requests
    q = engine.normal(n, loop.Q_HEADS, loop.DIM).bfloat16()
    starts, contexts = loop.int32(range(n + 1)), loop.int32([t - 1 for t in engine.lens])
    batch = K.make_batch(starts, contexts, n, 1, max(engine.lens))
    out = torch.empty_like(q)
    ws = torch.empty(max(16, K.kvx_attend_workspace(engine.view, batch, loop.Q_HEADS)), dtype=torch.uint8,
                     device="cuda")
    K.kvx_attend(engine.view, batch, engine.scores, 1, q, out, None, ws)
    for r in range(n):
        k = rows_of(engine, loop, 1, 0, r).double().repeat_interleave(loop.GROUP, 1).permute(1, 0, 2)
        v = rows_of(engine, loop, 1, 1, r).double().repeat_interleave(loop.GROUP, 1).permute(1, 0, 2)
        p = torch.softmax((k @ q[r].double()[:, :, None])[..., 0] * loop.DIM ** -0.5, -1)
        want = (p[:, None] @ v)[:, 0]
        size = (p[:, None] @ v.abs())[:, 0]
        # two roundings to bf16 (weights, output), scores to 1e-5
        assert ((out[r].double() - want).abs() <= size * (2.1 * 2.0 ** -8 + 1e-4) + 1e-7).all()


def test_eviction_keeps_what_was_weighed(loop):
    """After a step's weights: what stays are the first slots, the last, and the heaviest."""
    engine = loop.Engine([120, 50], pages=12, seed=3)
    engine.step(8)
    before = [rows_of(engine, loop, 0, 0, r).clone() for r in range(2)]
    weights = engine.weights.clone()
    lens = list(engine.lens)
    kept = engine.evict()
    assert engine.lens == [min(t, loop.BUDGET) for t in lens]
    for h in range(loop.HEADS):
        slots = kept[0, 0, h].long()
        assert slots[:loop.SINK].tolist() == list(range(loop.SINK))
        assert slots[-loop.RECENT:].tolist() == list(range(lens[0] - loop.RECENT, lens[0]))
        gone = sorted(set(range(lens[0])) - set(slots.tolist()))
        middle = slots[loop.SINK:-loop.RECENT]
        assert weights[0, 0, h, middle].min() >= weights[0, 0, h, gone].max()
        assert torch.equal(rows_of(engine, loop, 0, 0, 0)[:, h], before[0][slots, h])
    assert torch.equal(rows_of(engine, loop, 0, 0, 1), before[1])
