"""kvx_verify against its definition in 64 bits, token for token: chains and trees,
with and without a draft's logits, greedy requests, every type, rows of any length and
alignment, rows that are no distribution; and that what comes out is distributed as
the target."""
import math
import random

import pytest
import torch

import serving_reference as ref

pytestmark = pytest.mark.gpu
TORCH = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def K():
    import paper_2509_17542_amd as K
    return K


def int32(v):
    return torch.tensor(v, dtype=torch.int32).cuda()


class Problem:
    """Requests of `new` tokens; a peaked target, a draft near it, drafted tokens from the draft."""

    def __init__(self, new, vocab=300, dtype="bf16", tree=False, draft=False, distinct=False, temperatures=None,
                 seed=0, pad=0, shift=0, peak=8.0, near=0.9, siblings=4):
        g = torch.Generator().manual_seed(seed)
        rnd = random.Random(seed)
        self.new, self.vocab, self.distinct, self.dtype = list(new), vocab, distinct, dtype
        N = sum(new)
        self.tokens_n = N
        self.starts = [sum(new[:r]) for r in range(len(new) + 1)]
        width = vocab + pad
        target = torch.randn((N, width), generator=g) * 2
        if N:
            target.scatter_add_(1, torch.randint(0, vocab, (N, 4), generator=g), peak * torch.rand((N, 4), generator=g))
        small = near * target + (1 - near) * 6 * torch.randn((N, width), generator=g)
        # a buffer that starts `shift` elements late: rows aligned to their elements only
        def rows(x):
            flat = torch.zeros(N * width + shift, dtype=TORCH[dtype])
            flat[shift:] = x.to(TORCH[dtype]).flatten()
            d = flat.cuda()
            return flat[shift:].view(N, width)[:, :vocab], d[shift:].view(N, width)[:, :vocab]
        self.logits, self.d_logits = rows(target)
        self.draft, self.d_draft = rows(small) if draft else (None, None)
        self.temperatures = temperatures
        self.parents = None
        if tree:
            self.parents = []
            for n in new:
                p = [7]
                for i in range(1, n):
                    p.append(rnd.randint(max(0, i - siblings), i - 1))
                self.parents += p[:n]
        source = small if draft else small + 0.0
        self.tokens = []
        for r, n in enumerate(new):
            taken = {}
            for i in range(n):
                u = self.starts[r] + (0 if i == 0 else i - 1 if not tree else self.parents[self.starts[r] + i])
                z = source[u, :vocab].clone()
                if distinct or not draft:
                    for x in taken.get(u, []):
                        z[x] = -math.inf
                if draft and z.max() > -math.inf:
                    x = int(torch.multinomial(torch.softmax(z, 0), 1, generator=g))
                else:
                    x = int(z.argmax())
                taken.setdefault(u, []).append(x)
                self.tokens.append(x)
        self.uniforms = torch.rand(N, generator=g)
        self.samples = torch.rand(len(new), generator=g)

    def run(self, K, a_stride=None, stream=None, max_tokens=None):
        R = len(self.new)
        if a_stride is None:
            a_stride = max(max(self.new, default=1), 1)
        t = None if self.temperatures is None else torch.tensor(self.temperatures, dtype=torch.float32).cuda()
        drafts = K.make_drafts(int32(self.starts), int32(self.tokens), max_tokens or max(max(self.new, default=1), 1),
                               self.vocab, parents=None if self.parents is None else int32(self.parents),
                               temperatures=t, distinct=self.distinct)
        nbytes = K.kvx_verify_workspace(drafts, self.draft is not None)
        ws = torch.full((max(nbytes, 16),), 0xFF, dtype=torch.uint8, device="cuda")
        acc = torch.full((R, a_stride), 99, dtype=torch.int32, device="cuda")
        counts, nxt = (torch.full((R,), 99, dtype=torch.int32, device="cuda") for _ in range(2))
        K.kvx_verify(drafts, self.d_logits, self.d_draft, self.uniforms.cuda(), self.samples.cuda(), acc, counts, nxt,
                     ws, stream=stream)
        return acc.cpu(), counts.cpu(), nxt.cpu()

    def want(self, a_stride=None):
        out = []
        for r in range(len(self.new)):
            a, b = self.starts[r], self.starts[r + 1]
            out.append(ref.verify(self.tokens[a:b], None if self.parents is None else self.parents[a:b],
                                  self.logits[a:b], None if self.draft is None else self.draft[a:b],
                                  1.0 if self.temperatures is None else self.temperatures[r], self.uniforms[a:b],
                                  self.samples[r], self.distinct, a_stride))
        return out

    def check(self, K, a_stride=None):
        acc, counts, nxt = self.run(K, a_stride)
        for r, (path, token) in enumerate(self.want(a_stride)):
            assert int(counts[r]) == len(path), (r, counts[r], path)
            assert acc[r].tolist() == path + [-1] * (acc.shape[1] - len(path)), r
            assert int(nxt[r]) == token, (r, nxt[r], token)
        return counts


KINDS = [dict(), dict(tree=True), dict(draft=True), dict(tree=True, draft=True),
         dict(tree=True, draft=True, distinct=True)]


@pytest.mark.parametrize("kind", KINDS, ids=str)
@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
def test_types(K, kind, dtype):
    p = Problem([5, 1, 9, 0, 16, 2], dtype=dtype, seed=1, **kind)
    p.check(K)


@pytest.mark.parametrize("kind", KINDS, ids=str)
@pytest.mark.parametrize("vocab,pad", [(1, 0), (2, 0), (7, 1), (64, 0), (255, 0), (4095, 0), (4096, 0), (4097, 3),
                                       (8192, 8), (50257, 0)])
def test_vocabularies(K, kind, vocab, pad):
    """Rows of any length, aligned to their elements only, of one part and of several."""
    for seed in range(2):
        Problem([6, 3], vocab=vocab, pad=pad, shift=1, seed=10 + seed, dtype="fp16", peak=12.0, **kind).check(K)


@pytest.mark.parametrize("kind", KINDS, ids=str)
@pytest.mark.parametrize("near", [0.2, 0.7, 0.98])
def test_acceptance(K, kind, near):
    """Drafts far from the target and near it: short paths and long ones."""
    p = Problem([12] * 60, vocab=500, seed=int(100 * near), near=near, peak=15.0, **kind)
    counts = p.check(K)
    # paths of every kind: some end at once, some go far; near drafts, drawn, mostly do
    assert (counts == 1).any() or near == 0.98
    if near == 0.98:
        assert counts.max() >= 3 and (p.draft is None or counts.float().mean() > 2.0)


@pytest.mark.parametrize("kind", KINDS, ids=str)
def test_temperatures(K, kind):
    """Greedy and hot requests side by side; NaN and negative ones are greedy, tiny ones nearly so."""
    t = [0.0, 0.3, 1.0, 2.0, math.nan, -1.0, 1e-3, 1e-12, 100.0, 1e30, math.inf, 1e-30]
    Problem([6] * len(t), seed=3, temperatures=t, **kind).check(K)


@pytest.mark.parametrize("kind", KINDS, ids=str)
def test_path_cut(K, kind):
    """A path of a_stride tokens ends there: its last counts as a leaf."""
    for most in (1, 2, 3):
        Problem([9] * 20, seed=4, near=0.98, peak=15.0, **kind).check(K, a_stride=most)


def test_one_token_only(K):
    """Requests without drafted tokens: the next token alone."""
    Problem([1] * 40, vocab=1000, seed=5).check(K)
    Problem([1] * 40, vocab=1000, seed=5, draft=True).check(K)


def test_no_requests(K):
    p = Problem([0, 0, 0])
    acc, counts, nxt = p.run(K)
    assert (acc == -1).all() and (counts == 0).all() and (nxt == -1).all()
    p = Problem([0, 0, 0], draft=True)
    acc, counts, nxt = p.run(K)
    assert (acc == -1).all() and (counts == 0).all() and (nxt == -1).all()


@pytest.mark.parametrize("kind", KINDS, ids=str)
def test_ties_and_infinities(K, kind):
    """Equal logits, masked ones (-infinity), a row of one token."""
    p = Problem([6, 6, 6, 6], vocab=5000, seed=6, temperatures=[0.0, 1.0, 1.0, 0.0], **kind)
    for x in (p.logits, p.d_logits):
        x[:, 2000:4500] = -math.inf
        x[3:9] = x[3:9].round()
        x[12] = -math.inf
        x[12, 4700] = 3.0
        x[20, :] = 1.0
    p.check(K)


@pytest.mark.parametrize("kind", KINDS, ids=str)
@pytest.mark.parametrize("bad", [math.nan, math.inf, "none"])
def test_rows_that_are_no_distribution(K, kind, bad):
    p = Problem([5, 5, 5, 5], vocab=5000, seed=7, near=0.98, temperatures=[1.0, 0.0, 1.0, 1.0], **kind)
    for x in (p.logits, p.d_logits):
        for row in (0, 6, 12):
            if bad == "none":
                x[row] = -math.inf
            else:
                x[row, 4321] = bad
    if p.draft is not None:
        for x in (p.draft, p.d_draft):
            x[15, 17] = math.nan
            x[13] = -math.inf
    acc, counts, nxt = p.run(K)
    assert nxt[0] == -1 and counts[0] == 1
    p.check(K)


def test_tokens_out_of_range(K):
    """Token ids outside the vocabulary and parents that are none: never accepted, never read."""
    for kind in KINDS:
        p = Problem([6, 6, 6], seed=8, near=0.98, **kind)
        p.tokens[1], p.tokens[8], p.tokens[13] = -1, p.vocab, 2 ** 31 - 1
        if p.parents is not None:
            p.parents[4], p.parents[10], p.parents[16] = -1, 4, 2 ** 30
            p.parents[9] = 5
        p.check(K)


@pytest.mark.parametrize("kind", KINDS[1:2] + KINDS[3:], ids=str)
def test_same_token_twice(K, kind):
    """Siblings that are the same token."""
    for seed in range(6):
        p = Problem([10] * 6, vocab=20, seed=20 + seed, siblings=10, **kind)
        for r in range(6):
            for i in range(2, 10):
                if i % 3 == 0:
                    p.tokens[10 * r + i] = p.tokens[10 * r + i - 1]
        p.check(K)


def test_uniforms_at_the_ends(K):
    """Random numbers of 0 and of the largest below 1, samples too."""
    for kind in KINDS:
        p = Problem([7] * 12, vocab=6000, seed=9, **kind)
        p.uniforms[::2], p.uniforms[1::2] = 0.0, 1.0 - 2.0 ** -24
        p.samples[::2], p.samples[1::2] = 0.0, 1.0 - 2.0 ** -24
        p.check(K)


@pytest.mark.parametrize("kind", [dict(), dict(tree=True), dict(draft=True), dict(tree=True, draft=True, distinct=True)],
                         ids=str)
def test_largest_request(K, kind):
    """1024 tokens of one request."""
    p = Problem([1024, 3], vocab=40, seed=11, near=0.99, siblings=3, **kind)
    p.check(K)


@pytest.mark.parametrize("dtype", ["fp16", "fp32"])
@pytest.mark.parametrize("kind", KINDS, ids=str)
def test_many_logits(K, kind, dtype):
    """17 million logits, whose last rows are summed again: requests without tokens (whose share of the
    workspace nobody fills), greedy and nearly greedy ones, paths cut, rows that are no distribution."""
    new = [5, 0, 9, 16, 0, 2, 1, 30, 24, 28, 0]
    t = [1.0, 1.0, 0.0, 0.5, 0.7, 2.0, 0.0, 1.0, 1e-12, 0.9, 1.0]
    p = Problem(new, vocab=150001, dtype=dtype, seed=21, near=0.98, peak=15.0, temperatures=t, shift=1, **kind)
    assert p.logits.numel() >= 1 << 24
    p.check(K)
    p.check(K, a_stride=2)
    for x in (p.logits, p.d_logits):
        x[p.starts[3]] = -math.inf
        x[p.starts[7], 77] = math.nan
        x[p.starts[9], 5:] = -math.inf
    p.check(K)


def test_wide_star(K):
    """Hundreds of children of one token."""
    for draft in (False, True):
        p = Problem([300], vocab=900, seed=12, tree=True, draft=draft, near=0.1, peak=2.0)
        p.parents[1:] = [0] * 299
        p.tokens[1:] = torch.randperm(900, generator=torch.Generator().manual_seed(1))[:299].tolist()
        p.uniforms[:] = 0.9999
        p.check(K)


def test_bounds_cut(K):
    """A request longer on the device than max_tokens is cut to it."""
    p = Problem([8, 8], seed=13, near=0.98)
    acc, counts, nxt = p.run(K, max_tokens=3)
    q = Problem([8, 8], seed=13, near=0.98)
    for r in range(2):
        a = q.starts[r]
        path, token = ref.verify(q.tokens[a:a + 3], None, q.logits[a:a + 3], None, 1.0, q.uniforms[a:a + 3], q.samples[r])
        assert int(counts[r]) == len(path) and int(nxt[r]) == token


@pytest.mark.parametrize("kind", KINDS, ids=str)
def test_distribution(K, kind):
    """The first two tokens that come out (accepted or next), over 40000 requests whose drafted tokens are
    drawn anew, are distributed as the target: each frequency within five standard deviations."""
    V, R, n = 6, 40000, 4
    g = torch.Generator(device="cuda").manual_seed(14)
    target = torch.tensor([2.0, 1.0, 0.3, -0.5, 0.0, 1.5], device="cuda")
    small = torch.tensor([0.5, 1.5, 0.0, 0.7, -1.0, 1.2], device="cuda")
    logits = target.expand(R * n, V).contiguous()
    draft = small.expand(R * n, V).contiguous() if kind.get("draft") else None
    # token 0 the root, then a chain of three, or two children of the root and one of the first of them
    parents = int32([0, 0, 0, 1] * R) if kind.get("tree") else None
    q = torch.softmax(small, 0)
    if kind.get("draft"):
        x = torch.multinomial(q.expand(R * 4, V), 1, replacement=True, generator=g).view(R, 4)
        if kind.get("distinct"):
            two = torch.multinomial(q.expand(R, V), 2, replacement=False, generator=g)
            x[:, 1:3] = two
    else:
        x = small.argsort(descending=True)[:4].expand(R, 4).clone()
    drafts = K.make_drafts(torch.arange(0, R * n + 1, n, dtype=torch.int32, device="cuda"), x.int().flatten().contiguous(),
                           n, V, parents=parents, distinct=kind.get("distinct", False))
    ws = torch.empty(K.kvx_verify_workspace(drafts, draft is not None), dtype=torch.uint8, device="cuda")
    acc = torch.empty((R, n), dtype=torch.int32, device="cuda")
    counts, nxt = (torch.empty(R, dtype=torch.int32, device="cuda") for _ in range(2))
    K.kvx_verify(drafts, logits, draft, torch.rand(R * n, generator=g, device="cuda"),
                 torch.rand(R, generator=g, device="cuda"), acc, counts, nxt, ws)
    p = torch.softmax(target.double(), 0).cpu()
    first = torch.where(counts > 1, x.gather(1, acc[:, 1:2].clamp(min=0).long())[:, 0], nxt.long())
    seen = torch.bincount(first, minlength=V).double().cpu() / R
    assert ((seen - p).abs() <= 5 * (p * (1 - p) / R).sqrt()).all(), (seen, p)
    some = counts > 1
    second = torch.where(counts > 2, x.gather(1, acc[:, 2:3].clamp(min=0).long())[:, 0], nxt.long())[some]
    seen = torch.bincount(second, minlength=V).double().cpu() / len(second)
    assert ((seen - p).abs() <= 5 * (p * (1 - p) / len(second)).sqrt()).all(), (seen, p)


def test_graph_replays(K):
    """Captured on a stream of its own; replayed with other logits, tokens and random numbers, eager calls
    of another batch between."""
    p = Problem([5, 3, 8], vocab=5000, seed=15, tree=True, draft=True)
    other = Problem([4, 4], vocab=300, seed=16)
    R = 3
    drafts = K.make_drafts(int32(p.starts), int32(p.tokens), 8, 5000, parents=int32(p.parents))
    ws = torch.empty(K.kvx_verify_workspace(drafts, True), dtype=torch.uint8, device="cuda")
    acc = torch.zeros((R, 8), dtype=torch.int32, device="cuda")
    counts, nxt = (torch.zeros(R, dtype=torch.int32, device="cuda") for _ in range(2))
    u, s = p.uniforms.cuda(), p.samples.cuda()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        K.kvx_verify(drafts, p.d_logits, p.d_draft, u, s, acc, counts, nxt, ws, stream=stream)
        stream.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            K.kvx_verify(drafts, p.d_logits, p.d_draft, u, s, acc, counts, nxt, ws, stream=stream)
    for seed in range(4):
        q = Problem([5, 3, 8], vocab=5000, seed=30 + seed, tree=True, draft=True)
        p.d_logits.copy_(q.d_logits)
        p.d_draft.copy_(q.d_draft)
        drafts.keep[1].copy_(int32(q.tokens))
        drafts.keep[2].copy_(int32(q.parents))
        u.copy_(q.uniforms)
        s.copy_(q.samples)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for r, (path, token) in enumerate(q.want()):
            assert acc[r].tolist() == path + [-1] * (8 - len(path)) and int(nxt[r]) == token
        other.check(K)


def test_two_at_once(K):
    """Two streams, a workspace each."""
    a, b = (Problem([6] * 30, vocab=20000, seed=s, tree=True, draft=True) for s in (17, 18))
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for p, s in zip((a, b), streams):
        with torch.cuda.stream(s):
            got.append(p.run(K, stream=s))
    for p, (acc, counts, nxt) in zip((a, b), got):
        for r, (path, token) in enumerate(p.want()):
            assert acc[r].tolist() == path + [-1] * (6 - len(path)) and int(nxt[r]) == token
