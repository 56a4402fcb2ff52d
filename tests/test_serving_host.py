"""Host side of kvx_fetch, kvx_verify and the 4-bit cache (runs without a GPU):
entry points exported and bound, bad arguments refused before anything is launched,
calls of too many threads too, and the binding's refusals."""
import ctypes
import os
import re

import pytest
import torch

import test_operators_host as host
from conftest import ROOT
from test_operators_host import GOOD

K = pytest.importorskip("paper_2509_17542_amd")


def test_every_declared_function_is_exported():
    with open(os.path.join(ROOT, "include", "kvx_serve.h")) as f:
        names = sorted(set(re.findall(r"^(?:kvx_status|int32_t)\s+(kvx_\w+)\s*\(", f.read(), re.M)))
    assert names == sorted(K.SERVING) and len(names) == 4
    assert all(hasattr(K._lib, n) for n in names)
    assert K.kvx_serve_version() == K.SERVE_VERSION == 1


def four(**over):
    return host.cache(**{**dict(dtype=K.E2M1, scales=GOOD), **over})


def fetch(c=None, b=None, layer=0, dtype=K.BF16, k=GOOD, ks=256, v=GOOD, vs=256):
    c, b = c or host.cache(), b or host.batch()
    return K._lib.kvx_fetch(c.ref, b.ref, layer, dtype, k, ks, v, vs, None)


def drafts(**over):
    f = dict(num_requests=3, total_tokens=5, max_tokens=4, vocab=100, distinct=0, reserved=0, token_starts=GOOD,
             tokens=GOOD, parents=None, temperatures=None)
    f.update(over)
    d = K.kvx_drafts(**f)
    d.ref = ctypes.addressof(d)
    return d


def verify(d=None, dtype=K.BF16, logits=GOOD, stride=100, draft=None, ds=0, u=GOOD, s=GOOD, acc=GOOD, a_stride=4,
           counts=GOOD, nxt=GOOD, ws=GOOD, nbytes=1 << 40):
    d = d or drafts()
    return K._lib.kvx_verify(d.ref, dtype, logits, stride, draft, ds, u, s, acc, a_stride, counts, nxt, ws, nbytes, None)


def test_four_bit_caches_are_refused():
    for call in (host.attend, host.append, host.evict, host.commit, fetch):
        for dim in (16, 48, 80, 112):
            assert call(c=four(head_dim=dim)) == K.EINVAL
        assert call(c=four(head_dim=288)) == K.EUNSUPPORTED
        assert call(c=four(scales=None)) == K.EINVAL
        assert call(c=four(scales=GOOD + 4)) == K.EINVAL
        assert call(c=four(cache=None)) == K.EINVAL


def test_fetch_is_refused():
    for over in host.SHAPES:
        assert fetch(c=host.cache(**over)) == K.EINVAL
    assert fetch(layer=2) == K.EINVAL and fetch(layer=-1) == K.EINVAL
    assert fetch(dtype=K.E4M3FN) == K.EINVAL and fetch(dtype=K.E2M1) == K.EINVAL and fetch(dtype=0) == K.EINVAL
    for bad in (None, GOOD + 8):
        assert fetch(k=bad) == K.EINVAL and fetch(v=bad) == K.EINVAL
    for stride in (255, 248, -256):
        assert fetch(ks=stride) == K.EINVAL and fetch(vs=stride) == K.EINVAL
    for over in (dict(max_tokens=0), dict(max_context=0), dict(token_starts=None), dict(contexts=None)):
        assert fetch(b=host.batch(**over)) == K.EINVAL
    assert fetch(b=host.batch(total_tokens=0), k=None) == K.OK
    assert fetch(c=host.cache(num_requests=0), k=None) == K.OK
    assert fetch(b=host.batch(total_tokens=1 << 28)) == K.EUNSUPPORTED


@pytest.mark.parametrize("over", [
    dict(num_requests=-1), dict(total_tokens=-1), dict(max_tokens=0), dict(max_tokens=1025), dict(vocab=0),
    dict(vocab=(1 << 24) + 1), dict(token_starts=None), dict(tokens=None)], ids=str)
def test_drafts_are_refused(over):
    assert verify(d=drafts(**over)) == K.EINVAL
    assert K.kvx_last_error()


@pytest.mark.parametrize("over", [
    dict(dtype=0), dict(dtype=K.E4M3FN), dict(dtype=7), dict(logits=None), dict(logits=GOOD + 1), dict(stride=99),
    dict(dtype=6, logits=GOOD + 2), dict(draft=GOOD, ds=99), dict(draft=GOOD + 1, ds=100), dict(u=None), dict(s=None),
    dict(acc=None), dict(a_stride=0), dict(counts=None), dict(nxt=None), dict(ws=None), dict(ws=GOOD + 8),
    dict(nbytes=0)], ids=str)
def test_verify_is_refused(over):
    assert verify(**over) == K.EINVAL


def test_nothing_to_verify():
    assert verify(d=drafts(num_requests=0), logits=None, ws=None, acc=None) == K.OK


def test_workspace():
    def size(draft, **over):
        out = ctypes.c_uint64()
        assert K._lib.kvx_verify_workspace(drafts(**over).ref, draft, ctypes.byref(out)) == K.OK
        return out.value
    assert size(0) == 16 * 5
    assert size(0, vocab=4097) == 2 * 16 * 5
    assert size(1) >= 2 * 16 * 5 + 8 * 5 + 8 * 3 + 4 * 3
    assert size(1, num_requests=0) == 0
    assert K._lib.kvx_verify_workspace(drafts().ref, 0, None) == K.EINVAL
    need = size(1)
    assert verify(draft=GOOD, ds=100, nbytes=need - 1) == K.EINVAL


def test_too_many_threads():
    # parts: 4 a workgroup of 256; a request's workgroup has 512 threads
    assert verify(d=drafts(total_tokens=1 << 26)) == K.EUNSUPPORTED
    assert verify(d=drafts(num_requests=1 << 23)) == K.EUNSUPPORTED
    assert verify(d=drafts(total_tokens=1 << 25), draft=GOOD, ds=100) == K.EUNSUPPORTED
    assert verify(d=drafts(total_tokens=1 << 23, parents=GOOD), draft=GOOD, ds=100) == K.EUNSUPPORTED
    assert "threads" in K.kvx_last_error()


@pytest.mark.skipif(torch.cuda.device_count() > 0, reason="the pointers are none: only where no device can take them")
def test_good_calls_reach_the_device():
    assert verify() == K.EDEVICE and verify(draft=GOOD, ds=100) == K.EDEVICE
    assert verify(dtype=6) == K.EDEVICE
    assert fetch() == K.EDEVICE and fetch(c=four()) == K.EDEVICE
    assert host.append(c=four()) == K.EDEVICE and host.commit(c=four()) == K.EDEVICE
    assert host.evict(c=four()) == K.EDEVICE


@pytest.mark.parametrize("requests,context", [(1, 100), (3, 100), (3, 16384), (600, 16384)])
@pytest.mark.parametrize("over", [dict(), dict(head_dim=256), dict(num_kv_heads=1), dict(num_kv_heads=7, head_dim=96)],
                         ids=str)
def test_attend_plans_of_a_four_bit_cache(requests, context, over):
    """The sums of ranges hold a row of statistics and elements each; planes of more groups than 32 bits
    number are for the other kernel, whose sums are of splits."""
    shape = dict(num_requests=requests, bt_stride=1024, **over)
    heads = 4 * shape.get("num_kv_heads", 4)
    b = host.batch(total_tokens=requests, max_tokens=1, max_context=context)
    nbytes = ctypes.c_uint64()

    def workspace(c):
        assert K._lib.kvx_attend_workspace(c.ref, b.ref, heads, ctypes.byref(nbytes)) == K.OK
        return nbytes.value

    small, large = four(**shape), four(num_blocks=1 << 32, **shape)
    dim = shape.get("head_dim", 64)
    if context == 100 or requests >= 512:
        assert workspace(small) == 0             # a workgroup to each
    else:
        assert workspace(small) >= 16 * (2 + dim) * 4 and workspace(small) < 1 << 27
    splits = workspace(large) / (4 * ((requests * heads + 3) // 4) * (2 + dim) * 4)
    filled = requests * heads // 4 >= 768        # with a workgroup to each
    assert splits == int(splits) and (splits == 0) == (context == 100 or filled)
    for c in (small, large):
        if workspace(c):
            assert host.attend(c=c, b=b, heads=heads, qs=heads * dim, os_=heads * dim, nbytes=nbytes.value - 1) == K.EINVAL
        if torch.cuda.device_count() == 0:
            assert host.attend(c=c, b=b, heads=heads, qs=heads * dim, os_=heads * dim) == K.EDEVICE


def test_binding_refuses_layouts():
    table = torch.zeros((1, 4), dtype=torch.int32)
    codes = torch.zeros((1, 2, 3, 16, 2, 32), dtype=torch.uint8)
    scales = torch.zeros((1, 2, 3, 16, 2, 2), dtype=torch.uint8)
    with pytest.raises(ValueError, match="scales must be given"):
        K.make_cache(codes[..., :0], None, table, dtype=K.E2M1)
    with pytest.raises(ValueError, match="device"):
        K.make_cache(codes, scales, table, dtype=K.E2M1)
    empty = codes[:, :, :0]
    with pytest.raises(ValueError, match="scales must be"):
        K.make_cache(empty, scales[:, :, :0, :, :, :1], table, dtype=K.E2M1)
    with pytest.raises(ValueError, match="uint8 or float8_e8m0fnu"):
        K.make_cache(empty, scales[:, :, :0].float(), table, dtype=K.E2M1)
    with pytest.raises(ValueError, match="groups of 32"):
        K.make_cache(empty[..., :24], scales[:, :, :0], table, dtype=K.E2M1)
    with pytest.raises(ValueError, match="token_starts"):
        K.make_drafts(torch.zeros((0,), dtype=torch.int32), torch.zeros((0,), dtype=torch.int32), 4, 100)
    with pytest.raises(ValueError, match="device"):
        K.make_drafts(torch.zeros((2,), dtype=torch.int32), torch.zeros((3,), dtype=torch.int32), 4, 100)


def test_binding_refuses_logits():
    d = drafts(total_tokens=3)
    from paper_2509_17542_amd import serving
    with pytest.raises(ValueError, match="must be"):
        serving._logits(torch.zeros((3, 99)), "logits", d, None)
    with pytest.raises(ValueError, match="device"):
        serving._logits(torch.zeros((3, 100)), "logits", d, None)
