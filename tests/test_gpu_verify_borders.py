"""kvx_verify next to the borders of its decisions: temperatures and random numbers for which a
64-bit decision is clear, and one by exponentials of fewer bits is not.

An exponential is off by 1.4e-13 (the polynomial) and 3 roundings of its argument, 4e-16
of it in nats: below 1.6e-13 up to 30 nats.  So is an accepted token's probability; what the next token
goes by has half of it in the tail, and a quarter of that error in the border.  Borders are
taken from 3e-13 (1e-13 for the next token) to ten times that."""
import numpy as np
import pytest
import torch

from test_gpu_verify import KINDS, TORCH, Problem, int32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def K():
    import paper_2509_17542_amd as K
    return K


def near_borders(distance, vocab, many, least, seed, relative):
    """(temperature, fp32 number next to the probability, whether it is below): of token 1 (relative)
    or token 0, the others being `distance` below token 0."""
    rng, found = np.random.default_rng(seed), []
    centre = distance / np.log(vocab - 1) if not relative else 1.0
    while len(found) < many:
        t = (centre * rng.uniform(0.9, 1.1, 400000)).astype(np.float32)
        w = np.exp(-np.longdouble(distance) / t.astype(np.longdouble))
        p = (w if relative else np.longdouble(1)) / (1 + (vocab - 1) * w)
        s = p.astype(np.float32)
        off = (p - s.astype(np.longdouble)) / (p if relative else 1)
        for i in np.flatnonzero((abs(off) > least) & (abs(off) < 10 * least)):
            found.append((float(t[i]), float(s[i]), bool(off[i] > 0)))
    return found[:many]


def verify(K, logits, tokens, n, temperatures, uniforms, samples, draft=None):
    R, vocab = logits.shape[0] // n, logits.shape[1]
    drafts = K.make_drafts(torch.arange(0, R * n + 1, n, dtype=torch.int32, device="cuda"), int32(tokens), n, vocab,
                           temperatures=torch.tensor(temperatures, dtype=torch.float32).cuda())
    ws = torch.full((max(16, K.kvx_verify_workspace(drafts, draft is not None)),), 0xFF, dtype=torch.uint8, device="cuda")
    acc = torch.full((R, n), 99, dtype=torch.int32, device="cuda")
    counts, nxt = (torch.full((R,), 99, dtype=torch.int32, device="cuda") for _ in range(2))
    u, s = (torch.tensor(x, dtype=torch.float32).cuda() for x in (uniforms, samples))
    K.kvx_verify(drafts, logits, draft, u, s, acc, counts, nxt, ws)
    return counts.tolist(), nxt.tolist()


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("vocab,distance", [(20001, 6.0), (20001, 13.0), (4000, 8.5)])
def test_next_token(K, vocab, distance, dtype):
    """The first token has about half of the row, which a sample passes or does not."""
    near = near_borders(distance, vocab, 60, 1e-13, vocab, False)
    logits = torch.full((60, vocab), 2.0, dtype=TORCH[dtype], device="cuda")
    logits[:, 0] += distance
    _, nxt = verify(K, logits, [0] * 60, 1, [t for t, _, _ in near], [0.0] * 60, [s for _, s, _ in near])
    assert nxt == [0 if below else 1 for _, _, below in near]


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("distance", [2.0, 11.0, 27.0])
def test_accepted(K, distance, dtype):
    """A drafted token of a small probability, whose uniform number is next to that; alike with a
    draft that was sure of it."""
    vocab = 2
    near = near_borders(distance, vocab, 60, 3e-13, int(distance), True)
    logits = torch.zeros((120, vocab), dtype=TORCH[dtype], device="cuda")
    logits[:, 0] += distance
    sure = torch.zeros_like(logits)
    sure[:, 0] = float("-inf")
    u = sum(([0.0, s] for _, s, _ in near), [])
    for draft in (None, sure):
        counts, _ = verify(K, logits, [0, 1] * 60, 2, [t for t, _, _ in near], u, [0.5] * 60, draft)
        assert counts == [2 if below else 1 for _, _, below in near]


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
def test_accepted_in_a_large_call(K, dtype):
    """The same decisions among 2^24 logits and more: as in a call of the request alone."""
    vocab, distance, many = 20001, 10.0, 420
    near = near_borders(distance, vocab, many, 3e-13, 5, True)
    logits = torch.zeros((2 * many, vocab), dtype=TORCH[dtype], device="cuda")
    assert logits.numel() >= 1 << 24
    logits[:, 0] += distance
    t, u = [t for t, _, _ in near], sum(([0.0, s] for _, s, _ in near), [])
    counts, nxt = verify(K, logits, [0, 1] * many, 2, t, u, [0.7] * many)
    assert counts == [2 if below else 1 for _, _, below in near]
    for r in range(0, many, 30):
        alone = verify(K, logits[2 * r:2 * r + 2], [0, 1], 2, t[r:r + 1], u[2 * r:2 * r + 2], [0.7])
        assert alone == (counts[r:r + 1], nxt[r:r + 1])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kind", KINDS, ids=str)
def test_alone_and_among_others(K, kind, dtype):
    """A request's path and next token do not depend on how many others are in the call."""
    new = [6, 30, 1, 16, 24, 9, 30]
    p = Problem(new, vocab=150001, dtype=dtype, seed=31, near=0.97, peak=15.0, **kind)
    assert p.logits.numel() >= 1 << 24
    p.check(K)
    _, counts, nxt = p.run(K)
    for r in (0, 2, 5):
        a, b = p.starts[r], p.starts[r + 1]
        one = Problem([new[r]], vocab=4, dtype=dtype, seed=1, **kind)
        one.vocab, one.tokens, one.parents = p.vocab, p.tokens[a:b], None if p.parents is None else p.parents[a:b]
        one.d_logits, one.d_draft = p.d_logits[a:b], None if p.draft is None else p.d_draft[a:b]
        one.uniforms, one.samples = p.uniforms[a:b], p.samples[r:r + 1]
        _, c, n = one.run(K)
        assert (int(c), int(n)) == (int(counts[r]), int(nxt[r]))
