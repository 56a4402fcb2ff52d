"""What follows an eviction: new tokens appended behind the kept slots, attention and
weights over them with a window, a prefix and a bias by distance, which go by slots."""
import pytest
import torch

import operator_reference as ref
from operator_reference import Problem
from test_gpu_attend import check, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def K():
    import paper_2509_17542_amd as K
    return K


@pytest.mark.parametrize("cache", ["bf16", "e4m3fn"])
@pytest.mark.parametrize("new", [[1, 2], [30, 17]])
def test_bias_and_window_go_by_slots(K, new, cache):
    before = Problem(new=[0, 0], ctx=[300, 50], cache=cache, spare=40)
    view, _, _ = before.gpu(K)
    w = torch.rand((1, 2, before.heads, 300), device="cuda")
    kept = torch.zeros((1, 2, before.heads, 100), dtype=torch.int32, device="cuda")
    lens = torch.zeros(2, dtype=torch.int32, device="cuda")
    K.kvx_evict(view, 0, 1, torch.tensor([300, 50], dtype=torch.int32).cuda(), 300, 100, 4, 30, w, w, kept, lens)
    assert lens.tolist() == [100, 50]
    p = Problem(new=new, ctx=[100, 50], cache=cache, window=60, prefix=[4, 4], slopes=True)
    k, v = (torch.randn((p.tokens, p.heads, p.dim), device="cuda").bfloat16() for _ in range(2))
    starts = torch.tensor(p.starts, dtype=torch.int32).cuda()
    batch = K.make_batch(starts, lens, p.tokens, p.max_tokens, p.max_context)
    rope = K.make_rope(torch.zeros(0, device="cuda"), [0], torch.zeros((1, p.tokens), dtype=torch.int32, device="cuda"))
    K.kvx_append(view, batch, rope, 0, None, k, v, None)
    p.table, p.blocks = before.table, before.blocks
    p.cache = before.d_cache.cpu()
    p.scales = before.d_scales.cpu() if before.scales is not None else None
    out, lse, (view, batch, scores, _) = run(K, p)
    check(p, out, lse)
    start = torch.zeros((2, p.heads, p.max_context))
    weights = start.cuda()
    K.kvx_weigh(view, batch, scores, 0, p.q.cuda(), lse, weights)
    want, tol = ref.weigh(p, lse.cpu(), start)
    assert ((weights.double().cpu() - want).abs() <= tol).all()
