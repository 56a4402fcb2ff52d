"""Host side of the decode operators (runs without a GPU): the entry points that
include/kvx_ops.h declares are exported and bound, bad arguments come back as
status codes before anything is launched, calls with nothing to do succeed, and
the binding refuses tensors that a launch would read or write outside of."""
import ctypes
import os
import re

import pytest
import torch

from conftest import ROOT

K = pytest.importorskip("paper_2509_17542_amd")

GOOD = 0x10000            # stands for a device pointer: never read on the host


def declared():
    with open(os.path.join(ROOT, "include", "kvx_ops.h")) as f:
        text = f.read()
    return sorted(set(re.findall(r"^(?:kvx_status|int32_t)\s+(kvx_\w+)\s*\(", text, re.M)))


def test_every_declared_operator_is_exported():
    names = declared()
    assert names == sorted(K.OPERATORS) and len(names) == 7
    for n in names:
        assert hasattr(K._lib, n), n
    assert K.kvx_ops_version() == K.OPS_VERSION == 1
    assert K.kvx_abi_version() == 9             # the conversions' ABI is what it was


def cache(**over):
    f = dict(num_layers=2, num_kv_heads=4, head_dim=64, dtype=K.BF16, block_size=16, num_requests=3,
             bt_stride=8, reserved=0, num_blocks=32, cache=GOOD, scales=None, block_table=GOOD)
    f.update(over)
    c = K.kvx_cache(**f)
    c.ref = ctypes.addressof(c)
    return c


def batch(**over):
    f = dict(total_tokens=5, max_tokens=3, max_context=100, tree_stride=0, token_starts=GOOD,
             contexts=GOOD, positions=None, tree=None)
    f.update(over)
    b = K.kvx_batch(**f)
    b.ref = ctypes.addressof(b)
    return b


def scores(**over):
    f = dict(scale=0.125, softcap=0.0, window=0, reserved=0, slopes=None, prefix=None)
    f.update(over)
    s = K.kvx_scores(**f)
    s.ref = ctypes.addressof(s)
    return s


def rope(pairs=32, sections=(32,), interleaved=0, **over):
    f = dict(pairs=pairs, interleaved=interleaved, num_axes=len(sections),
             sections=(ctypes.c_int32 * 4)(*sections), reserved=0, inv_freq=GOOD, positions=GOOD)
    f.update(over)
    r = K.kvx_rope(**f)
    r.ref = ctypes.addressof(r)
    return r


def attend(c=None, b=None, s=None, layer=0, dtype=K.BF16, heads=8, q=GOOD, qs=512, out=GOOD, os_=512,
           lse=None, ws=GOOD, nbytes=1 << 40):
    c, b, s = c or cache(), b or batch(), s or scores()
    return K._lib.kvx_attend(c.ref, b.ref, s.ref, layer, dtype, heads, q, qs, out, os_, lse, ws, nbytes, None)


def weigh(c=None, b=None, s=None, layer=0, dtype=K.BF16, heads=8, q=GOOD, qs=512, lse=GOOD, w=GOOD, ws=100):
    c, b, s = c or cache(), b or batch(), s or scores()
    return K._lib.kvx_weigh(c.ref, b.ref, s.ref, layer, dtype, heads, q, qs, lse, w, ws, None)


def append(c=None, b=None, r=None, layer=0, dtype=K.BF16, heads=8, q=GOOD, qs=512, k=GOOD, ks=256, v=GOOD,
           vs=256, out=GOOD, os_=512):
    c, b, r = c or cache(), b or batch(), r or rope()
    return K._lib.kvx_append(c.ref, b.ref, r.ref, layer, dtype, heads, q, qs, k, ks, v, vs, out, os_, None)


def evict(c=None, layer0=0, n=2, lens=GOOD, max_len=100, budget=50, sink=4, recent=10, w=GOOD, w_out=GOOD,
          ws=100, kept=GOOD, new=GOOD + 64):
    c = c or cache()
    return K._lib.kvx_evict(c.ref, layer0, n, lens, max_len, budget, sink, recent, w, w_out, ws, kept, new, None)


def commit(c=None, layer0=0, n=2, ctx=GOOD, acc=GOOD, stride=4, counts=GOOD, new=GOOD + 64):
    c = c or cache()
    return K._lib.kvx_commit(c.ref, layer0, n, ctx, acc, stride, counts, new, None)


SHAPES = [dict(num_layers=0), dict(num_kv_heads=0), dict(head_dim=0), dict(head_dim=60), dict(block_size=0),
          dict(num_blocks=0), dict(dtype=0), dict(dtype=9), dict(num_requests=-1), dict(bt_stride=-1),
          dict(dtype=K.E4M3FN, head_dim=72, scales=GOOD)]


@pytest.mark.parametrize("over", SHAPES, ids=str)
def test_cache_shapes_are_refused(over):
    for call in (attend, weigh, append, evict, commit):
        assert call(c=cache(**over)) == K.EINVAL
        assert K.kvx_last_error()


def test_sizes_that_are_not_built_are_refused():
    for call in (attend, weigh, append, evict, commit):
        assert call(c=cache(head_dim=264)) == K.EUNSUPPORTED
        assert call(c=cache(num_kv_heads=2000)) == K.EUNSUPPORTED
        assert call(c=cache(num_blocks=1 << 58)) == K.EUNSUPPORTED
    big = dict(bt_stride=1 << 30, block_size=16)
    assert attend(c=cache(**big), b=batch(max_context=(1 << 30) + 1)) == K.EUNSUPPORTED
    assert evict(c=cache(**big), max_len=(1 << 30) + 1, ws=1 << 31) == K.EUNSUPPORTED
    assert attend(heads=4 * 1025, qs=64 * 4 * 1025, os_=64 * 4 * 1025) == K.EUNSUPPORTED
    assert attend(dtype=K.FP16) == K.EUNSUPPORTED       # a bf16 cache, fp16 queries
    assert weigh(dtype=K.FP16) == K.EUNSUPPORTED


@pytest.mark.parametrize("over", [
    dict(total_tokens=-1), dict(max_tokens=0), dict(max_tokens=65537), dict(max_context=0),
    dict(max_context=129), dict(token_starts=None), dict(contexts=None), dict(tree=GOOD, tree_stride=0),
    dict(tree=GOOD, tree_stride=1, max_tokens=65)], ids=str)
def test_batches_are_refused(over):
    for call in (attend, weigh, append):
        assert call(b=batch(**over)) == K.EINVAL


@pytest.mark.parametrize("over", [
    dict(scale=float("nan")), dict(scale=float("inf")), dict(softcap=-1.0), dict(softcap=float("inf")),
    dict(softcap=float("nan")), dict(window=-1)], ids=str)
def test_scores_are_refused(over):
    assert attend(s=scores(**over)) == K.EINVAL
    assert weigh(s=scores(**over)) == K.EINVAL


def test_arguments_are_refused():
    for call in (attend, weigh, append):
        assert call(layer=-1) == K.EINVAL and call(layer=2) == K.EINVAL
        assert call(dtype=K.E4M3FN) == K.EINVAL
        assert call(q=None) == K.EINVAL and call(q=GOOD + 8) == K.EINVAL
        assert call(qs=511) == K.EINVAL and call(qs=504) == K.EINVAL
        assert call(c=cache(cache=None)) == K.EINVAL
        assert call(c=cache(cache=GOOD + 4)) == K.EINVAL
        assert call(c=cache(block_table=None)) == K.EINVAL
        assert call(c=cache(scales=GOOD)) == K.EINVAL
        assert call(c=cache(dtype=K.E4M3FN)) == K.EINVAL
    for call in (attend, weigh):
        assert call(heads=0) == K.EINVAL and call(heads=6) == K.EINVAL
    assert attend(out=None) == K.EINVAL and attend(out=GOOD + 2) == K.EINVAL and attend(os_=256) == K.EINVAL
    # 64 requests of up to 100 slots have no need of splits, 5000 slots do
    many = cache(bt_stride=400)
    assert attend(c=many, b=batch(max_context=5000), ws=None) == K.EINVAL
    assert attend(c=many, b=batch(max_context=5000), nbytes=100) == K.EINVAL
    assert attend(c=many, b=batch(max_context=5000), ws=GOOD + 8) == K.EINVAL
    assert weigh(lse=None) == K.EINVAL and weigh(w=None) == K.EINVAL and weigh(ws=99) == K.EINVAL
    assert append(k=None) == K.EINVAL and append(v=GOOD + 8) == K.EINVAL and append(ks=255) == K.EINVAL
    assert append(out=None) == K.EINVAL and append(heads=-1) == K.EINVAL
    for bad in (rope(pairs=33, sections=(33,)), rope(pairs=-1), rope(num_axes=0), rope(num_axes=5),
                rope(sections=(16, 8)), rope(sections=(40, -8)), rope(inv_freq=None), rope(positions=None)):
        assert append(r=bad) == K.EINVAL
    assert evict(layer0=1) == K.EINVAL and evict(n=-1) == K.EINVAL
    assert evict(max_len=129) == K.EINVAL and evict(max_len=-1) == K.EINVAL
    assert evict(budget=0, sink=0, recent=0) == K.EINVAL and evict(sink=-1) == K.EINVAL
    assert evict(sink=45, recent=10) == K.EINVAL and evict(recent=2 ** 31 - 1, sink=2 ** 31 - 1) == K.EINVAL
    assert evict(ws=99) == K.EINVAL
    for name in ("lens", "w", "w_out", "kept", "new"):
        assert evict(**{name: None}) == K.EINVAL
    assert evict(new=GOOD) == K.EINVAL
    assert commit(layer0=1) == K.EINVAL and commit(stride=-1) == K.EINVAL and commit(new=GOOD) == K.EINVAL
    for name in ("ctx", "acc", "counts", "new"):
        assert commit(**{name: None}) == K.EINVAL


def test_null_structs_are_refused():
    c, b, s = cache(), batch(), scores()
    out = ctypes.c_uint64()
    assert K._lib.kvx_attend(None, b.ref, s.ref, 0, 2, 8, GOOD, 512, GOOD, 512, None, None, 0, None) == K.EINVAL
    assert K._lib.kvx_attend(c.ref, None, s.ref, 0, 2, 8, GOOD, 512, GOOD, 512, None, None, 0, None) == K.EINVAL
    assert K._lib.kvx_attend(c.ref, b.ref, None, 0, 2, 8, GOOD, 512, GOOD, 512, None, None, 0, None) == K.EINVAL
    assert K._lib.kvx_append(c.ref, b.ref, None, 0, 2, 8, GOOD, 512, GOOD, 256, GOOD, 256, GOOD, 512, None) == K.EINVAL
    assert K._lib.kvx_attend_workspace(c.ref, b.ref, 8, None) == K.EINVAL
    assert K._lib.kvx_attend_workspace(c.ref, b.ref, 7, ctypes.byref(out)) == K.EINVAL
    assert K._lib.kvx_evict(None, 0, 1, GOOD, 1, 1, 0, 0, GOOD, GOOD, 1, GOOD, GOOD, None) == K.EINVAL
    assert K._lib.kvx_commit(None, 0, 1, GOOD, GOOD, 1, GOOD, GOOD, None) == K.EINVAL


def test_nothing_to_do_inspects_no_pointer():
    none = dict(cache=None, block_table=None)
    empty = batch(total_tokens=0, token_starts=None, contexts=None)
    for call in (attend, weigh, append):
        assert call(c=cache(**none), b=empty, q=None) == K.OK
        assert call(c=cache(num_requests=0, **none), q=None) == K.OK
    assert evict(c=cache(num_requests=0, **none), lens=None) == K.OK
    assert evict(n=0, lens=None) == K.OK
    assert commit(c=cache(num_requests=0, **none), ctx=None) == K.OK


def test_workspace_holds_the_splits():
    """None for one split; else a sum and a pair of statistics per split, token and query head."""
    def need(c, b, heads):
        out = ctypes.c_uint64()
        assert K._lib.kvx_attend_workspace(c.ref, b.ref, heads, ctypes.byref(out)) == K.OK
        return out.value
    assert need(cache(), batch(max_context=100), 8) == 0
    assert need(cache(), batch(total_tokens=0), 8) == 0
    c = cache(bt_stride=1000)
    got = need(c, batch(max_context=2048), 8)
    assert got % (5 * 8 * (64 + 2) * 4) == 0 and got // (5 * 8 * (64 + 2) * 4) >= 2
    assert need(c, batch(max_context=16000), 8) > got


# ---- the binding -----------------------------------------------------------------

def test_host_tensors_are_refused():
    shape = (1, 2, 4, 16, 2, 64)
    table = torch.zeros((1, 4), dtype=torch.int32)
    with pytest.raises(ValueError, match="device"):
        K.make_cache(torch.zeros(shape, dtype=torch.bfloat16), None, table)
    with pytest.raises(ValueError, match="device"):
        K.make_batch(torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), 1, 1, 1)
    with pytest.raises(ValueError, match="device"):
        K.make_scores(1.0, slopes=torch.zeros(4))
    with pytest.raises(ValueError, match="device"):
        K.make_rope(torch.zeros(4), [4], torch.zeros((1, 3), dtype=torch.int32))


def test_shapes_are_refused_by_the_binding():
    table = torch.zeros((1, 4), dtype=torch.int32)
    with pytest.raises(ValueError, match="layers"):
        K.make_cache(torch.zeros((2, 4, 16, 2, 64), dtype=torch.bfloat16), None, table)
    with pytest.raises(ValueError, match="dtype"):
        K.make_cache(torch.zeros((1, 2, 4, 16, 2, 64), dtype=torch.uint8), None, table)
    with pytest.raises(ValueError, match="dtype"):
        K.make_cache(torch.zeros((1, 2, 4, 16, 2, 64), dtype=torch.float32), None, table)
    with pytest.raises(ValueError, match="token_starts"):
        K.make_batch(torch.zeros(3, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), 1, 1, 1)
    with pytest.raises(ValueError, match="axes"):
        K.make_rope(torch.zeros(4), [1, 1, 1, 1, 0], torch.zeros((5, 3), dtype=torch.int32))
    with pytest.raises(ValueError, match="per section"):
        K.make_rope(torch.zeros(4), [2, 2], torch.zeros((1, 3), dtype=torch.int32))


def test_names_are_those_of_the_package():
    assert {"kvx_attend", "make_cache", "make_scores"} <= set(K._OPERATOR_NAMES)
    for n in K._OPERATOR_NAMES:
        assert getattr(K, n) is not None
    with pytest.raises(AttributeError):
        K.kvx_no_such_thing
