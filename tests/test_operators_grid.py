"""Calls of more threads than one launch may have (HIP takes fewer than 2^32,
workgroups times their size) are refused, whichever of a call's launches it is,
before the first of them; one workgroup fewer is not.  Runs without a GPU: a call
that passes all checks then ends at the missing device, before any launch."""
import pytest
import torch

import test_operators_host as host

K = pytest.importorskip("paper_2509_17542_amd")

MANY = [
    # name, the call for n, the least n that is too many
    ("append", lambda n: host.append(b=host.batch(total_tokens=n)), 1 << 24),
    ("select_short", lambda n: host.evict(c=host.cache(num_layers=1, num_kv_heads=1, num_requests=n), n=1), 1 << 23),
    ("select_heads", lambda n: host.evict(c=host.cache(num_layers=2, num_kv_heads=4, num_requests=n), n=2), 1 << 20),
    ("select_long", lambda n: host.evict(c=host.cache(num_layers=1, num_kv_heads=1, num_requests=n, bt_stride=1000), n=1,
                                         max_len=4097, ws=4097), 1 << 22),
    ("commit", lambda n: host.commit(c=host.cache(num_layers=1, num_requests=n), n=1), 1 << 24),
    ("commit_none", lambda n: host.commit(c=host.cache(num_layers=1, num_requests=n), n=0), 1 << 24),
    ("commit_planes", lambda n: host.commit(c=host.cache(num_layers=5, num_requests=n), n=5), 1 << 23),
    ("few", lambda n: host.attend(c=host.cache(num_kv_heads=1, num_requests=n), heads=1), 1 << 24),
    ("few_splits", lambda n: host.attend(c=host.cache(num_kv_heads=2, num_requests=n, bt_stride=400), heads=2,
                                         b=host.batch(max_context=2048)), 1 << 21),
    ("rows_64", lambda n: host.attend(c=host.cache(num_kv_heads=1, num_requests=n), heads=1,
                                      b=host.batch(max_tokens=40)), 1 << 25),
    ("rows_tiles", lambda n: host.attend(c=host.cache(num_kv_heads=1, num_requests=n), heads=1,
                                         b=host.batch(max_tokens=129)), 1 << 23),
    ("join", lambda n: host.attend(c=host.cache(bt_stride=400), b=host.batch(total_tokens=n, max_context=5000)), 1 << 23),
    ("join_many", lambda n: host.attend(c=host.cache(bt_stride=2000), b=host.batch(total_tokens=n, max_context=33 * 512)),
     1 << 21),
    ("weigh", lambda n: host.weigh(c=host.cache(num_requests=n)), 1 << 22),
    ("weigh_tiles", lambda n: host.weigh(c=host.cache(num_requests=n, bt_stride=20), b=host.batch(max_context=129),
                                         ws=129), 1 << 21),
    ("weigh_held", lambda n: host.weigh(c=host.cache(num_requests=n, bt_stride=20),
                                        b=host.batch(max_context=256, max_tokens=9), ws=256), 1 << 22),
]


@pytest.mark.parametrize("call,n", [m[1:] for m in MANY], ids=[m[0] for m in MANY])
def test_too_many_threads(call, n):
    for more in (n, n + 1, 2 * n):
        assert call(more) == K.EUNSUPPORTED
        assert "threads" in K.kvx_last_error()


@pytest.mark.skipif(torch.cuda.device_count() > 0, reason="the pointers are none: only where no device can take them")
@pytest.mark.parametrize("call,n", [m[1:] for m in MANY], ids=[m[0] for m in MANY])
def test_one_fewer(call, n):
    assert call(n - 1) == K.EDEVICE
