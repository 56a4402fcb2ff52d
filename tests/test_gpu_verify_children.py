"""kvx_verify where a token has many children and the draft's logits are given: the refusals one after
the other, as the definition makes them, and what they cost."""
import statistics

import pytest
import torch

import serving_reference as ref
from test_gpu_verify import TORCH, int32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def K():
    import paper_2509_17542_amd as K
    return K


class Star:
    """Requests whose first token has all the others as children, drawn from the draft."""

    def __init__(self, children, vocab, dtype, distinct, requests, seed, spread=1.0, temperature=1.0):
        g = torch.Generator().manual_seed(seed)
        self.n, self.vocab, self.distinct, self.t = children + 1, vocab, distinct, temperature
        N = requests * self.n
        target = 2 * torch.randn((N, vocab), generator=g)
        small = target + spread * torch.randn((N, vocab), generator=g)
        self.logits, self.draft = target.to(TORCH[dtype]), small.to(TORCH[dtype])
        self.tokens, self.uniforms, self.samples = [], [], torch.rand(requests, generator=g)
        for r in range(requests):
            q = torch.softmax(self.draft[r * self.n].double() / temperature, 0)
            x = torch.multinomial(q, children, replacement=not distinct, generator=g).tolist()
            self.tokens.append([0] + x)
            # refused until far down the list, most of them
            self.uniforms.append(1.0 - 0.5 ** (2 + (6 * r + 13) % 20) * torch.rand(self.n, generator=g))
        self.uniforms = [u.clamp(max=1 - 2.0 ** -24) for u in self.uniforms]
        self.parents = [-1] + [0] * children

    def call(self, K):
        R, n = len(self.tokens), self.n
        drafts = K.make_drafts(torch.arange(0, R * n + 1, n, dtype=torch.int32, device="cuda"),
                               int32(sum(self.tokens, [])), n, self.vocab, parents=int32(self.parents * R),
                               temperatures=torch.full((R,), self.t, device="cuda"), distinct=self.distinct)
        ws = torch.full((K.kvx_verify_workspace(drafts, True),), 0xFF, dtype=torch.uint8, device="cuda")
        acc = torch.full((R, n), 99, dtype=torch.int32, device="cuda")
        counts, nxt = (torch.full((R,), 99, dtype=torch.int32, device="cuda") for _ in range(2))
        args = (drafts, self.logits.cuda(), self.draft.cuda(), torch.cat(self.uniforms).cuda(), self.samples.cuda(), acc,
                counts, nxt, ws)
        return lambda: K.kvx_verify(*args), (acc, counts, nxt)

    def want(self, r):
        a = slice(r * self.n, (r + 1) * self.n)
        return ref.verify(self.tokens[r], self.parents, self.logits[a], self.draft[a], self.t, self.uniforms[r],
                          self.samples[r], self.distinct)


CASES = [(2, 5000, 20), (3, 300, 20), (40, 5000, 20), (300, 3000, 8), (1023, 4099, 3)]


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("distinct", [False, True])
@pytest.mark.parametrize("children,vocab,requests", CASES)
def test_refusals(K, children, vocab, requests, distinct, dtype):
    p = Star(children, vocab, dtype, distinct, requests, children, temperature=0.8)
    call, (acc, counts, nxt) = p.call(K)
    call()
    for r in range(requests):
        path, token = p.want(r)
        assert acc[r].tolist() == path + [-1] * (p.n - len(path)) and int(nxt[r]) == token, r


@pytest.mark.parametrize("distinct", [False, True])
def test_cost_of_children(K, distinct):
    """Four times the children take four times the refusals over the row, not sixteen times the work."""
    times = []
    for children in (128, 512):
        p = Star(children, 8192, "bf16", distinct, 1, 3)
        p.uniforms[0][:] = 1 - 2.0 ** -24
        call, _ = p.call(K)
        call()
        took = []
        for _ in range(5):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            call()
            b.record()
            b.synchronize()
            took.append(a.elapsed_time(b))
        times.append(statistics.median(took))
    assert times[1] <= 8 * times[0], times
