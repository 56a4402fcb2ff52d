"""Python binding of the decode operators (include/kvx_ops.h): argument
marshalling only.

    view = make_cache(cache, scales, block_table)
    batch = make_batch(token_starts, contexts, total_tokens, max_tokens, max_context)
    kvx_append(view, batch, make_rope(...), layer, q, k, v, q_out)
    kvx_attend(view, batch, make_scores(...), layer, q, out, lse, workspace)
    kvx_weigh(view, batch, make_scores(...), layer, q, lse, weights)
    kvx_evict(view, layer0, num_layers, lens, max_len, budget, sink, recent, weights, ...)
    kvx_commit(view, layer0, num_layers, contexts, accepted, counts, new_lens)

Views, batches, ropes and scores hold the tensors that they were made of.  Every
tensor argument is checked (device, type, layout, size) before a launch, so that
a short one cannot become an access outside of it: ValueError, or KvxError with
the C call's status.
"""
from __future__ import annotations

import ctypes

import torch

from . import (BF16, E4M3FN, E5M2, FP16, _addr, _check, _i32, _lib, _need, _stream, _vp)

_i64 = ctypes.c_int64

OPS_VERSION = 1


class kvx_cache(ctypes.Structure):
    _fields_ = [("num_layers", _i32), ("num_kv_heads", _i32), ("head_dim", _i32), ("dtype", _i32),
                ("block_size", _i32), ("num_requests", _i32), ("bt_stride", _i32),
                ("reserved", _i32), ("num_blocks", _i64), ("cache", _vp), ("scales", _vp),
                ("block_table", _vp)]


class kvx_batch(ctypes.Structure):
    _fields_ = [("total_tokens", _i32), ("max_tokens", _i32), ("max_context", _i32),
                ("tree_stride", _i32), ("token_starts", _vp), ("contexts", _vp),
                ("positions", _vp), ("tree", _vp)]


class kvx_scores(ctypes.Structure):
    _fields_ = [("scale", ctypes.c_float), ("softcap", ctypes.c_float), ("window", _i32),
                ("reserved", _i32), ("slopes", _vp), ("prefix", _vp)]


class kvx_rope(ctypes.Structure):
    _fields_ = [("pairs", _i32), ("interleaved", _i32), ("num_axes", _i32), ("sections", _i32 * 4),
                ("reserved", _i32), ("inv_freq", _vp), ("positions", _vp)]


_SIGNATURES = {
    "kvx_append": [_vp, _vp, _vp, _i32, _i32, _i32, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _vp],
    "kvx_attend": [_vp, _vp, _vp, _i32, _i32, _i32, _vp, _i64, _vp, _i64, _vp, _vp, ctypes.c_uint64,
                   _vp],
    "kvx_attend_workspace": [_vp, _vp, _i32, ctypes.POINTER(ctypes.c_uint64)],
    "kvx_weigh": [_vp, _vp, _vp, _i32, _i32, _i32, _vp, _i64, _vp, _vp, _i64, _vp],
    "kvx_evict": [_vp, _i32, _i32, _vp, _i32, _i32, _i32, _i32, _vp, _vp, _i64, _vp, _vp, _vp],
    "kvx_commit": [_vp, _i32, _i32, _vp, _vp, _i32, _vp, _vp, _vp],
}
for _name, _args in _SIGNATURES.items():
    getattr(_lib, _name).restype = ctypes.c_int
    getattr(_lib, _name).argtypes = _args
_lib.kvx_ops_version.restype = ctypes.c_int32
_lib.kvx_ops_version.argtypes = []
if _lib.kvx_ops_version() != OPS_VERSION:
    raise ImportError(f"libkvx.so implements operators {_lib.kvx_ops_version()}, this binding "
                      f"{OPS_VERSION}: rebuild the library")

OPERATORS = tuple(sorted([*_SIGNATURES, "kvx_ops_version"]))

_CACHE_TYPES = {torch.float16: FP16, torch.bfloat16: BF16, torch.float8_e4m3fn: E4M3FN,
                torch.float8_e5m2: E5M2}
_ROW_TYPES = {torch.float16: FP16, torch.bfloat16: BF16}


def kvx_ops_version() -> int:
    return int(_lib.kvx_ops_version())


def make_cache(cache, scales, block_table, dtype=None) -> kvx_cache:
    """A decode rank's cache [layers][2][num_blocks][block_size][Hd][D] with its
    scales [layers][2][num_blocks][block_size][Hd] (None for 16 bits) and the
    block table [requests][stride] of the requests at hand.  `dtype` (E4M3FN,
    E5M2) says what codes held as uint8 are."""
    if cache.dim() != 6 or cache.shape[1] != 2:
        raise ValueError("cache must be [layers][2][num_blocks][block_size][heads][dim], not "
                         f"{list(cache.shape)}")
    kind = _CACHE_TYPES.get(cache.dtype)
    if kind is None:
        if cache.dtype != torch.uint8 or dtype not in (E4M3FN, E5M2):
            raise ValueError(f"a cache of {cache.dtype} needs dtype E4M3FN or E5M2 and uint8 codes")
        kind = dtype
    elif dtype not in (None, kind):
        raise ValueError(f"dtype {dtype} does not match {cache.dtype}")
    _need(cache, max(cache.nbytes, 1) if cache.numel() else 0, "cache")
    if (kind in (E4M3FN, E5M2)) != (scales is not None):
        raise ValueError("scales must be given exactly for an 8-bit cache")
    if scales is not None:
        if scales.shape != cache.shape[:-1]:
            raise ValueError(f"scales must be {list(cache.shape[:-1])}, not {list(scales.shape)}")
        _need(scales, scales.nbytes, "scales", torch.float32)
    if block_table.dim() != 2:
        raise ValueError("block_table must be [requests][stride]")
    _need(block_table, block_table.nbytes, "block_table", torch.int32)
    layers, _, blocks, size, heads, dim = cache.shape
    c = kvx_cache(layers, heads, dim, kind, size, block_table.shape[0], block_table.shape[1], 0,
                  blocks, _addr(cache), _addr(scales), _addr(block_table))
    c.ref = ctypes.addressof(c)
    c.keep = (cache, scales, block_table)
    return c


def make_batch(token_starts, contexts, total_tokens, max_tokens, max_context, positions=None,
               tree=None) -> kvx_batch:
    """The new tokens of the cache's requests: int32 device tensors
    token_starts [requests + 1], contexts [requests], positions [total_tokens]
    or None; `tree` int64 [total_tokens][words] (bit j of a token's words: it
    sees new token j of its request) or None for a chain.  max_tokens and
    max_context bound the lengths that the device tensors hold."""
    requests = contexts.shape[0]
    total_tokens = int(total_tokens)
    if contexts.dim() != 1 or token_starts.shape != (requests + 1,):
        raise ValueError("contexts must be [requests] and token_starts [requests + 1]")
    _need(contexts, 4 * requests, "contexts", torch.int32)
    _need(token_starts, 4 * requests + 4, "token_starts", torch.int32)
    if positions is not None:
        _need(positions, 4 * total_tokens, "positions", torch.int32)
    words = 0
    if tree is not None:
        if tree.dim() != 2:
            raise ValueError("tree must be [total_tokens][words]")
        words = tree.shape[1]
        _need(tree, 8 * total_tokens * words, "tree", torch.int64)
    b = kvx_batch(total_tokens, int(max_tokens), int(max_context), words, _addr(token_starts),
                  _addr(contexts), _addr(positions), _addr(tree))
    b.ref = ctypes.addressof(b)
    b.requests = requests
    b.tokens = total_tokens
    b.longest = int(max_context)
    b.keep = (token_starts, contexts, positions, tree)
    return b


def make_scores(scale, softcap=0.0, slopes=None, window=0, prefix=None) -> kvx_scores:
    """How scores are formed: slopes float32 [q_heads] (bias by distance), prefix
    int32 [requests] (slots that every token sees), device tensors or None."""
    if slopes is not None:
        _need(slopes, max(slopes.nbytes, 4), "slopes", torch.float32)
    if prefix is not None:
        _need(prefix, max(prefix.nbytes, 4), "prefix", torch.int32)
    s = kvx_scores(float(scale), float(softcap), int(window), 0, _addr(slopes), _addr(prefix))
    s.ref = ctypes.addressof(s)
    s.heads = slopes.numel() if slopes is not None else None
    s.requests = prefix.numel() if prefix is not None else None
    s.keep = (slopes, prefix)
    return s


def make_rope(inv_freq, sections, positions, interleaved=False) -> kvx_rope:
    """Rotary positions: inv_freq float32 [pairs], positions int32 [axes][tokens]
    (device tensors), `sections` the pairs of each axis."""
    sections = [int(n) for n in sections]
    if not 1 <= len(sections) <= 4:
        raise ValueError("one to four axes")
    if positions.dim() != 2 or positions.shape[0] != len(sections):
        raise ValueError("positions must be [axes][tokens], one row per section")
    pairs = inv_freq.numel()
    _need(inv_freq, 4 * pairs, "inv_freq", torch.float32)
    _need(positions, positions.nbytes, "positions", torch.int32)
    r = kvx_rope(pairs, int(bool(interleaved)), len(sections), (_i32 * 4)(*sections), 0,
                 _addr(inv_freq), _addr(positions))
    r.ref = ctypes.addressof(r)
    r.tokens = positions.shape[1]
    r.keep = (inv_freq, positions)
    return r


def _rows(x, what, tokens, dim, dtype):
    """A [tokens][heads][dim] device tensor whose heads are contiguous: its heads
    and the elements between tokens.  dtype None: float16 or bfloat16."""
    try:
        n, heads, d = x.shape
        s0, s1, s2 = x.stride()
    except ValueError:
        raise ValueError(f"{what} must be [{tokens}][heads][{dim}], not {list(x.shape)}") from None
    if n == tokens and d == dim and x.is_cuda and (s1 == dim or heads == 1) and s2 == 1 and \
            (x.dtype == dtype if dtype is not None else x.dtype in _ROW_TYPES):
        # one token, or none: no stride between tokens to speak of
        return heads, s0 if n > 1 else heads * dim
    if n != tokens or d != dim:
        raise ValueError(f"{what} must be [{tokens}][heads][{dim}], not {list(x.shape)}")
    if not x.is_cuda:
        raise ValueError(f"{what} must be a device tensor, not one on {x.device}")
    if x.dtype not in _ROW_TYPES or (dtype is not None and x.dtype != dtype):
        raise ValueError(f"{what} must be {dtype or 'float16 or bfloat16'}, not {x.dtype}")
    if n * heads == 0:
        return heads, heads * dim
    raise ValueError(f"{what}: the heads of a token must be contiguous")


def _match(view, batch, scores=None, q_heads=0):
    if batch.requests != view.num_requests:
        raise ValueError(f"a batch of {batch.requests} requests, a block table of {view.num_requests}")
    if scores is not None:
        if scores.heads not in (None, q_heads):
            raise ValueError(f"{scores.heads} slopes for {q_heads} query heads")
        if scores.requests is not None and scores.requests != view.num_requests:
            raise ValueError(f"{scores.requests} prefixes for {view.num_requests} requests")


def kvx_append(view, batch, rope, layer, q, k, v, q_out, stream=None) -> None:
    """q, q_out [tokens][q_heads][D] (q_out may be q; both None: keys and values
    only), k, v [tokens][Hd][D]; slices of a fused projection serve."""
    _match(view, batch)
    n, d, heads = batch.tokens, view.head_dim, view.num_kv_heads
    if rope.tokens != n:
        raise ValueError(f"positions of {rope.tokens} tokens, a batch of {n}")
    dtype = k.dtype
    (k_heads, ks), (v_heads, vs) = _rows(k, "k", n, d, None), _rows(v, "v", n, d, dtype)
    if k_heads != heads or v_heads != heads:
        raise ValueError(f"k and v must have the cache's {heads} heads")
    q_heads = qs = out_heads = os = 0
    if q is not None:
        q_heads, qs = _rows(q, "q", n, d, dtype)
        if q_out is None:
            raise ValueError("q_out must be given with q")
        out_heads, os = _rows(q_out, "q_out", n, d, dtype)
    if q_heads != out_heads:
        raise ValueError("q_out must have the heads of q")
    status = _lib.kvx_append(view.ref, batch.ref, rope.ref, layer, _ROW_TYPES[dtype], q_heads,
                             _addr(q), qs, k.data_ptr(), ks, v.data_ptr(), vs, _addr(q_out), os,
                             _stream(stream))
    if status:
        _check(status)


def kvx_attend_workspace(view, batch, q_heads: int) -> int:
    """Bytes of workspace that kvx_attend needs for these."""
    out = ctypes.c_uint64()
    _check(_lib.kvx_attend_workspace(view.ref, batch.ref, q_heads, ctypes.byref(out)))
    return out.value


def kvx_attend(view, batch, scores, layer, q, out, lse=None, workspace=None, stream=None) -> None:
    """q, out [tokens][q_heads][D]; lse float32 [tokens][q_heads] or None;
    workspace: a device tensor of kvx_attend_workspace bytes, or None for 0."""
    n, d = batch.tokens, view.head_dim
    dtype = q.dtype
    (q_heads, qs), (out_heads, os) = _rows(q, "q", n, d, None), _rows(out, "out", n, d, dtype)
    if out_heads != q_heads:
        raise ValueError("out must have the heads of q")
    _match(view, batch, scores, q_heads)
    if lse is not None:
        _need(lse, 4 * n * q_heads, "lse", torch.float32)
    nbytes = 0
    if workspace is not None:
        nbytes = workspace.nbytes
        _need(workspace, nbytes, "workspace")
    status = _lib.kvx_attend(view.ref, batch.ref, scores.ref, layer, _ROW_TYPES[dtype], q_heads,
                             q.data_ptr(), qs, out.data_ptr(), os, _addr(lse), _addr(workspace),
                             nbytes, _stream(stream))
    if status:
        _check(status)


def kvx_weigh(view, batch, scores, layer, q, lse, weights, stream=None) -> None:
    """lse float32 [tokens][q_heads] as kvx_attend gave it; weights float32
    [requests][Hd][stride], stride >= the batch's max_context."""
    n, d = batch.tokens, view.head_dim
    q_heads, qs = _rows(q, "q", n, d, None)
    _match(view, batch, scores, q_heads)
    _need(lse, 4 * n * q_heads, "lse", torch.float32)
    if weights.dim() != 3 or weights.shape[:2] != (view.num_requests, view.num_kv_heads):
        raise ValueError("weights must be [requests][heads][stride]")
    _need(weights, weights.nbytes, "weights", torch.float32)
    status = _lib.kvx_weigh(view.ref, batch.ref, scores.ref, layer, _ROW_TYPES[q.dtype], q_heads,
                            q.data_ptr(), qs, lse.data_ptr(), weights.data_ptr(), weights.shape[2],
                            _stream(stream))
    if status:
        _check(status)


def kvx_evict(view, layer0, num_layers, lens, max_len, budget, sink, recent, weights, weights_out,
              kept, new_lens, stream=None) -> None:
    """weights, weights_out float32 [num_layers][requests][Hd][stride] (may be one
    tensor), kept int32 [num_layers][requests][Hd][budget], lens and new_lens
    int32 [requests]."""
    R, heads = view.num_requests, view.num_kv_heads
    shape = (num_layers, R, heads)
    for x, what in ((weights, "weights"), (weights_out, "weights_out")):
        if x.dim() != 4 or x.shape[:3] != shape or x.shape[3] != weights.shape[3]:
            raise ValueError(f"{what} must be [{num_layers}][{R}][{heads}][stride]")
        _need(x, x.nbytes, what, torch.float32)
    if kept.shape != (*shape, budget):
        raise ValueError(f"kept must be [{num_layers}][{R}][{heads}][{budget}]")
    _need(kept, kept.nbytes, "kept", torch.int32)
    _need(lens, 4 * R, "lens", torch.int32)
    _need(new_lens, 4 * R, "new_lens", torch.int32)
    status = _lib.kvx_evict(view.ref, layer0, num_layers, lens.data_ptr(), max_len, budget, sink,
                            recent, weights.data_ptr(), weights_out.data_ptr(), weights.shape[3],
                            kept.data_ptr(), new_lens.data_ptr(), _stream(stream))
    if status:
        _check(status)


def kvx_commit(view, layer0, num_layers, contexts, accepted, counts, new_lens, stream=None) -> None:
    """accepted int32 [requests][stride] (ascending node numbers), contexts,
    counts and new_lens int32 [requests]."""
    R = view.num_requests
    if accepted.dim() != 2 or accepted.shape[0] != R:
        raise ValueError("accepted must be [requests][stride]")
    _need(accepted, accepted.nbytes, "accepted", torch.int32)
    for x, what in ((contexts, "contexts"), (counts, "counts"), (new_lens, "new_lens")):
        _need(x, 4 * R, what, torch.int32)
    status = _lib.kvx_commit(view.ref, layer0, num_layers, contexts.data_ptr(), accepted.data_ptr(),
                             accepted.shape[1], counts.data_ptr(), new_lens.data_ptr(),
                             _stream(stream))
    if status:
        _check(status)
