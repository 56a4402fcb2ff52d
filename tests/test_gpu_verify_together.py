"""Calls of kvx_verify that run at the same time: everything uploaded, then enqueued in turn on
streams of their own, nothing copied back in between."""
import pytest
import torch

from test_gpu_verify import KINDS, Problem, int32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def K():
    import paper_2509_17542_amd as K
    return K


class Call:
    """A problem's inputs, workspace and results on the device."""

    def __init__(self, K, p):
        R, self.p = len(p.new), p
        most = max(p.new)
        self.drafts = K.make_drafts(int32(p.starts), int32(p.tokens), most, p.vocab,
                                    parents=None if p.parents is None else int32(p.parents), distinct=p.distinct)
        nbytes = K.kvx_verify_workspace(self.drafts, p.draft is not None)
        self.space = torch.full((max(nbytes, 16),), 0xFF, dtype=torch.uint8, device="cuda")
        self.uniforms, self.samples = p.uniforms.cuda(), p.samples.cuda()
        self.accepted = torch.full((R, most), 99, dtype=torch.int32, device="cuda")
        self.counts, self.next = (torch.full((R,), 99, dtype=torch.int32, device="cuda") for _ in range(2))
        self.stream = torch.cuda.Stream()

    def enqueue(self, K):
        K.kvx_verify(self.drafts, self.p.d_logits, self.p.d_draft, self.uniforms, self.samples, self.accepted,
                     self.counts, self.next, self.space, stream=self.stream)

    def clear(self):
        for x in (self.accepted, self.counts, self.next):
            x.fill_(99)

    def check(self):
        for r, (path, token) in enumerate(self.p.want()):
            assert self.accepted[r].tolist() == path + [-1] * (self.accepted.shape[1] - len(path))
            assert int(self.counts[r]) == len(path) and int(self.next[r]) == token


@pytest.mark.parametrize("kind", KINDS, ids=str)
def test_streams(K, kind):
    """Three calls of other sizes, eight rounds of each: one's last kernels beside another's first."""
    calls = [Call(K, Problem(new, vocab=vocab, seed=seed, **kind))
             for new, vocab, seed in (([6] * 30, 20000, 41), ([9, 2, 30], 50257, 42), ([4] * 100, 5003, 43))]
    for _ in range(2):
        for c in calls:
            c.clear()
        torch.cuda.synchronize()
        for _ in range(8):
            for c in calls:
                c.enqueue(K)
        torch.cuda.synchronize()
        for c in calls:
            c.check()


@pytest.mark.parametrize("kind", KINDS[1:4:2], ids=str)
def test_graphs(K, kind):
    """Two captured calls, replayed on streams of their own at the same time, with other random numbers."""
    calls = [Call(K, Problem(new, vocab=vocab, seed=seed, **kind))
             for new, vocab, seed in (([6] * 30, 20000, 44), ([9, 2, 30], 50257, 45))]
    graphs = []
    torch.cuda.synchronize()
    for c in calls:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.stream(c.stream):
            c.enqueue(K)
            c.stream.synchronize()
            with torch.cuda.graph(graphs[-1], stream=c.stream):
                c.enqueue(K)
    for turn in range(3):
        g = torch.Generator().manual_seed(turn)
        for c in calls:
            c.clear()
            c.p.uniforms, c.p.samples = torch.rand(c.p.uniforms.shape, generator=g), torch.rand(c.p.samples.shape, generator=g)
            c.uniforms.copy_(c.p.uniforms)
            c.samples.copy_(c.p.samples)
        torch.cuda.synchronize()
        for _ in range(4):
            for c, graph in zip(calls, graphs):
                with torch.cuda.stream(c.stream):
                    graph.replay()
        torch.cuda.synchronize()
        for c in calls:
            c.check()
