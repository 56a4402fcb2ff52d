"""Python binding of include/kvx_serve.h (rows read back, verification of drafted
tokens): argument marshalling only, in the manner of operators.py.

    kvx_fetch(view, batch, layer, k, v)
    drafts = make_drafts(token_starts, tokens, max_tokens, vocab, parents, temperatures)
    kvx_verify(drafts, logits, draft, uniforms, samples, accepted, counts, next_tokens, workspace)
    kvx_commit(view, 0, layers, contexts, accepted, counts, new_lens)
"""
from __future__ import annotations

import ctypes

import torch

from . import BF16, FP16, _addr, _check, _i32, _lib, _need, _stream, _vp
from .operators import _ROW_TYPES, _match, _rows

_i64, _u64 = ctypes.c_int64, ctypes.c_uint64

SERVE_VERSION = 1
FP32 = 6


class kvx_drafts(ctypes.Structure):
    _fields_ = [("num_requests", _i32), ("total_tokens", _i32), ("max_tokens", _i32), ("vocab", _i32),
                ("distinct", _i32), ("reserved", _i32), ("token_starts", _vp), ("tokens", _vp),
                ("parents", _vp), ("temperatures", _vp)]


_SIGNATURES = {
    "kvx_fetch": [_vp, _vp, _i32, _i32, _vp, _i64, _vp, _i64, _vp],
    "kvx_verify": [_vp, _i32, _vp, _i64, _vp, _i64, _vp, _vp, _vp, _i32, _vp, _vp, _vp, _u64, _vp],
    "kvx_verify_workspace": [_vp, _i32, ctypes.POINTER(_u64)],
}
for _name, _args in _SIGNATURES.items():
    getattr(_lib, _name).restype = ctypes.c_int
    getattr(_lib, _name).argtypes = _args
_lib.kvx_serve_version.restype = ctypes.c_int32
_lib.kvx_serve_version.argtypes = []
if _lib.kvx_serve_version() != SERVE_VERSION:
    raise ImportError(f"libkvx.so implements version {_lib.kvx_serve_version()} of kvx_serve.h, this binding "
                      f"{SERVE_VERSION}: rebuild the library")

SERVING = tuple(sorted([*_SIGNATURES, "kvx_serve_version"]))

_LOGITS = {torch.float16: FP16, torch.bfloat16: BF16, torch.float32: FP32}


def kvx_serve_version() -> int:
    return int(_lib.kvx_serve_version())


def kvx_fetch(view, batch, layer, k, v, stream=None) -> None:
    """k, v [tokens][Hd][D] float16 or bfloat16, the heads of a token contiguous."""
    _match(view, batch)
    n, d = batch.tokens, view.head_dim
    dtype = k.dtype
    (k_heads, ks), (v_heads, vs) = _rows(k, "k", n, d, None), _rows(v, "v", n, d, dtype)
    if k_heads != view.num_kv_heads or v_heads != view.num_kv_heads:
        raise ValueError(f"k and v must have the cache's {view.num_kv_heads} heads")
    status = _lib.kvx_fetch(view.ref, batch.ref, layer, _ROW_TYPES[dtype], k.data_ptr(), ks, v.data_ptr(), vs,
                            _stream(stream))
    if status:
        _check(status)


def make_drafts(token_starts, tokens, max_tokens, vocab, parents=None, temperatures=None,
                distinct=False) -> kvx_drafts:
    """The drafted tokens of the requests, the first of each the one sampled last:
    int32 device tensors token_starts [requests + 1], tokens [total], parents
    [total] (numbers within the request) or None for a chain; temperatures float32
    [requests] or None; distinct: siblings were drawn without replacement."""
    if token_starts.dim() != 1 or token_starts.shape[0] < 1 or tokens.dim() != 1:
        raise ValueError("token_starts must be [requests + 1] and tokens [total]")
    requests, total = token_starts.shape[0] - 1, tokens.shape[0]
    _need(token_starts, 4 * requests + 4, "token_starts", torch.int32)
    _need(tokens, 4 * total, "tokens", torch.int32)
    if parents is not None:
        _need(parents, 4 * total, "parents", torch.int32)
    if temperatures is not None:
        _need(temperatures, 4 * requests, "temperatures", torch.float32)
    d = kvx_drafts(requests, total, int(max_tokens), int(vocab), int(bool(distinct)), 0, _addr(token_starts),
                   _addr(tokens), _addr(parents), _addr(temperatures))
    d.ref = ctypes.addressof(d)
    d.keep = (token_starts, tokens, parents, temperatures)
    return d


def kvx_verify_workspace(drafts, with_draft: bool) -> int:
    """Bytes of workspace that kvx_verify needs with or without the draft's logits."""
    out = _u64()
    _check(_lib.kvx_verify_workspace(drafts.ref, int(bool(with_draft)), ctypes.byref(out)))
    return out.value


def _logits(x, what, drafts, dtype):
    """A [tokens][vocab] device tensor whose rows are contiguous: the elements between rows."""
    if x.dim() != 2 or x.shape != (drafts.total_tokens, drafts.vocab):
        raise ValueError(f"{what} must be [{drafts.total_tokens}][{drafts.vocab}], not {list(x.shape)}")
    if not x.is_cuda:
        raise ValueError(f"{what} must be a device tensor, not one on {x.device}")
    if x.dtype not in _LOGITS or (dtype is not None and x.dtype != dtype):
        raise ValueError(f"{what} must be {dtype or 'float16, bfloat16 or float32'}, not {x.dtype}")
    if x.shape[0] <= 1:
        if x.numel() > 1 and x.stride(1) != 1 and x.shape[1] > 1:
            raise ValueError(f"{what}: the logits of a row must be contiguous")
        return drafts.vocab
    if (x.shape[1] > 1 and x.stride(1) != 1) or x.stride(0) < drafts.vocab:
        raise ValueError(f"{what}: the logits of a row must be contiguous, rows apart")
    return x.stride(0)


def kvx_verify(drafts, logits, draft, uniforms, samples, accepted, counts, next_tokens, workspace,
               stream=None) -> None:
    """logits, draft (or None) [tokens][vocab]; uniforms float32 [tokens], samples
    float32 [requests]; accepted int32 [requests][stride], counts and next_tokens
    int32 [requests]; workspace: a device tensor of kvx_verify_workspace bytes."""
    R, n = drafts.num_requests, drafts.total_tokens
    stride = _logits(logits, "logits", drafts, None)
    draft_stride = _logits(draft, "draft", drafts, logits.dtype) if draft is not None else 0
    _need(uniforms, 4 * n, "uniforms", torch.float32)
    _need(samples, 4 * R, "samples", torch.float32)
    if accepted.dim() != 2 or accepted.shape[0] != R:
        raise ValueError(f"accepted must be [{R}][stride]")
    _need(accepted, accepted.nbytes, "accepted", torch.int32)
    for x, what in ((counts, "counts"), (next_tokens, "next_tokens")):
        _need(x, 4 * R, what, torch.int32)
    nbytes = 0
    if workspace is not None:
        nbytes = workspace.nbytes
        _need(workspace, nbytes, "workspace")
    status = _lib.kvx_verify(drafts.ref, _LOGITS[logits.dtype], logits.data_ptr(), stride, _addr(draft),
                             draft_stride, _addr(uniforms), _addr(samples), accepted.data_ptr(),
                             accepted.shape[1], counts.data_ptr(), next_tokens.data_ptr(), _addr(workspace),
                             nbytes, _stream(stream))
    if status:
        _check(status)
