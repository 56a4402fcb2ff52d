"""kvx_verify of greedy requests: the first of the largest logits, wherever in the row it
lies -- at the ends of vocabularies whose last part is no whole number of 16-byte
vectors above all."""
import math

import pytest
import torch

from test_gpu_verify import KINDS, TORCH, Problem, int32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def K():
    import paper_2509_17542_amd as K
    return K


def verify(K, logits, tokens, n, draft=None, parents=None):
    """Greedy requests of n tokens each: paths, counts, next tokens."""
    R, vocab = logits.shape[0] // n, logits.shape[1]
    drafts = K.make_drafts(torch.arange(0, R * n + 1, n, dtype=torch.int32, device="cuda"), int32(tokens), n, vocab,
                           parents=None if parents is None else int32(parents),
                           temperatures=torch.zeros(R, device="cuda"))
    ws = torch.full((max(16, K.kvx_verify_workspace(drafts, draft is not None)),), 0xFF, dtype=torch.uint8, device="cuda")
    acc = torch.full((R, n), 99, dtype=torch.int32, device="cuda")
    counts, nxt = (torch.full((R,), 99, dtype=torch.int32, device="cuda") for _ in range(2))
    K.kvx_verify(drafts, logits, draft, torch.rand(R * n, device="cuda"), torch.rand(R, device="cuda"), acc, counts, nxt, ws)
    return acc.tolist(), counts.tolist(), nxt.tolist()


def rows_of(n, vocab, dtype, seed, pad=3):
    """Logits below 1, rows aligned to their elements only."""
    x = torch.rand((n, vocab + pad), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")
    return (x - 0.5).to(TORCH[dtype])[:, :vocab]


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("vocab", [1, 2, 3, 7, 9, 13, 300, 4097, 4105, 8191, 32001, 50257, 150001])
@pytest.mark.parametrize("draft", [False, True])
def test_largest_at_the_end(K, vocab, dtype, draft):
    """The largest logit at each of the last 9 tokens and of the first 9: as the next token, as a drafted
    one, and refusing a drafted one."""
    at = sorted({max(0, vocab - 9 + j) for j in range(9)} | set(range(min(9, vocab))))
    logits = rows_of(4 * len(at), vocab, dtype, vocab)
    tokens, want = [], []
    for i, x in enumerate(at):
        y = at[(i + 1) % len(at)]
        # a request whose drafted token is the largest's, and one whose is not
        logits[4 * i, x] = logits[4 * i + 1, y] = logits[4 * i + 2, x] = logits[4 * i + 3, y] = 5.0
        tokens += [0, x, 0, (x + 1) % vocab if vocab > 1 else -1]
        want += [([0, 1], 2, y), ([0, -1], 1, x)]
    got = verify(K, logits, tokens, 2, draft=rows_of(len(logits), vocab, dtype, 5) if draft else None)
    assert list(zip(*got)) == want


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
def test_many_logits(K, dtype):
    """The same in a call of 2^24 logits and more."""
    vocab = 150001
    at = [vocab - 9 + j for j in range(9)] + [0, 4095, 4096, vocab // 2] + [147455, 147456, 147457]
    logits = rows_of(128, vocab, dtype, 1)
    assert logits.numel() >= 1 << 24
    tokens, want = [], []
    for i in range(64):
        x, y = at[i % len(at)], at[(i + 1) % len(at)]
        logits[2 * i, x] = logits[2 * i + 1, y] = 5.0
        tokens += [0, x if i % 3 else (x + 1) % vocab]
        want.append(([0, 1], 2, y) if i % 3 else ([0, -1], 1, x))
    assert list(zip(*verify(K, logits, tokens, 2))) == want


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("vocab", [9, 13, 300, 4105, 50257])
def test_equal_largest(K, vocab, dtype):
    """Of equal largest logits the first, 0 and -0 among them: within the row's last vectors, and one
    ahead of them."""
    pairs = [(i, j) for j in range(max(0, vocab - 9), vocab) for i in {0, max(0, vocab - 10), j - 3, j - 1} if 0 <= i < j]
    logits = rows_of(len(pairs), vocab, dtype, 7) - 1.0
    for r, (i, j) in enumerate(pairs):
        logits[r, i], logits[r, j] = (5.0, 5.0) if r % 2 else (-0.0, 0.0)
    acc, counts, nxt = verify(K, logits, [0] * len(pairs), 1)
    assert nxt == [i for i, _ in pairs] and counts == [1] * len(pairs)


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("kind", KINDS, ids=str)
def test_masked_but_the_end(K, kind, dtype):
    """Rows whose last tokens alone are possible, greedy requests beside others."""
    for vocab in (29, 4099, 5003):
        p = Problem([6, 3, 5, 1], vocab=vocab, dtype=dtype, seed=vocab, shift=1, temperatures=[0.0, 1.0, 0.0, 0.0], **kind)
        for x in (p.logits, p.d_logits):
            x[:, :vocab - 3] = -math.inf
        for r, n in enumerate(p.new):
            for i in range(n):
                p.tokens[p.starts[r] + i] = vocab - 1 - (i + r) % 3
        p.check(K)
