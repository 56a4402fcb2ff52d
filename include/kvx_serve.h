/*
 * kvx_serve.h -- C ABI of two more operators of a decode engine, beside those of
 * kvx_ops.h:
 *
 *   kvx_fetch   rows of a cache read back into 16 bits
 *   kvx_verify  drafted tokens against the target's logits, from given random
 *               numbers: the path for kvx_commit and the token that follows it
 *
 * Ownership, streams, graphs and errors are those of kvx_ops.h: every buffer is
 * the caller's, the calls only launch kernels on the given hipStream_t, what the
 * device tensors hold is read when the kernels run, and results are the same in
 * every run.
 */
#ifndef KVX_SERVE_H
#define KVX_SERVE_H

#include "kvx_ops.h"

#ifdef __cplusplus
extern "C" {
#endif

#define KVX_SERVE_VERSION 1

int32_t kvx_serve_version(void);

/* Reads back what kvx_append wrote for the same batch: the keys and values of
 * slots contexts[r] .. contexts[r] + n_r - 1 of every request r (contexts 0: from
 * the first slot on) of layer `layer`, as values.
 *   dtype: KVX_FP16 or KVX_BF16, the type of k and v.
 *   k, v:  device; token t's heads are [Hd][D] at t * stride elements (strides are
 *          multiples of 8, pointers 16-byte aligned).
 * A value (8-bit codes: times their row's scale in fp32; 4-bit ones: times their
 * group's) is rounded once to dtype, to nearest even; of a cache of that type it is
 * copied.  A token whose slot has no page, or lies past max_context, and one past
 * its request's max_tokens, gives zeros; tokens of no request are not written.
 * KVX_EINVAL: NULL or misaligned pointers, sizes out of range, layer outside the
 * cache. */
kvx_status kvx_fetch(const kvx_cache *cache, const kvx_batch *batch, int32_t layer, int32_t dtype,
                     void *k, int64_t k_stride, void *v, int64_t v_stride, void *hip_stream);

/* The type of logits that have 32 bits; the others are KVX_FP16 and KVX_BF16. */
#define KVX_FP32 6

/* Drafted tokens of the requests: request r's are tokens token_starts[r] ..
 * token_starts[r + 1] - 1 of the flat axis.  The first of them is the one that the
 * request sampled last (the target has it as input now, it is not drafted any more);
 * the others are drafted, each to follow its parent. */
typedef struct {
    int32_t num_requests;       /* R >= 0 */
    int32_t total_tokens;       /* N >= 0 */
    int32_t max_tokens;         /* bound of a request's tokens, 1 .. 1024 */
    int32_t vocab;              /* V: 1 .. 2^24 */
    int32_t distinct;           /* 0: siblings were drawn independently, else without replacement */
    int32_t reserved;
    const int32_t *token_starts;/* device [R + 1], non-decreasing, within 0 .. N */
    const int32_t *tokens;      /* device [N]; one outside [0, V) has probability 0 */
    const int32_t *parents;     /* device [N] or NULL: the number within the request of the token that
                                 * a token follows, below its own (others are never reached).  The
                                 * request's first is not read.  NULL: a chain. */
    const float *temperatures;  /* device [R] or NULL (all 1).  0 (and anything below 2^-60, NaN
                                 * too): greedy; cut to 2^60. */
} kvx_drafts;

/* Verification.  Row i of the logits l is the target's after token i, p its
 * softmax(l / T); row i of the draft's logits, where given, is what the children of
 * token i were drawn from, q its softmax at the same temperature.  From a request's
 * first token on, at the last token accepted, with r = p and the children x of it in
 * ascending order:
 *   draft given:  x is accepted when uniform[x] * q(x) < r(x); otherwise r becomes
 *                 max(r - q, 0) / its sum (distinct: and q(x) 0, q divided by its sum);
 *   no draft:     (the tokens were not drawn: the likeliest ones, an n-gram's) x is
 *                 accepted when uniform[x] * sum of r < r(x); otherwise r(x) becomes 0.
 * Of a request with temperature 0 a child is accepted when its token is the first of
 * the row's largest logits.  After the last child is refused, and after a leaf, the
 * next token is drawn from r: the first v for which the sum of r(0) .. r(v) is above
 * sample[request] times the sum of all (greedy: that first largest; nothing left of
 * r: drawn from p).  So the accepted tokens and the next one are distributed as
 * the target's own.
 *   dtype:     KVX_FP16, KVX_BF16 or KVX_FP32, of both logits.
 *   logits, draft: device [N], rows `stride` elements apart, aligned to their
 *              elements; draft may be NULL.
 *   uniforms:  device fp32 [N], in [0, 1); the request's first is not read.
 *   samples:   device fp32 [R], in [0, 1).
 *   accepted:  device int32 [R][a_stride]: the path's numbers within the request,
 *              ascending from 0, then -1: kvx_commit's.  A path ends at its a_stride-th
 *              token, which then counts as a leaf.
 *   counts:    device int32 [R]: the path's length, 0 for a request of no tokens.
 *   next_tokens: device int32 [R]; -1 where there is none.
 *   workspace: device, >= kvx_verify_workspace bytes, 16-byte aligned; calls (and graphs) that may
 *              run at the same time need one each.
 * What tokens are accepted by and the next one is drawn by is summed in 64 bits, from
 * exponentials of 2e-13; it does not depend on the other requests of the call.  A row that has a NaN or +infinity, or nothing
 * but -infinity, is no distribution: after it all children are refused, and there is
 * no next token; where the draft's row is none, its children are refused and the next
 * token is drawn from p.
 * KVX_EINVAL: NULL pointers, sizes out of range, strides below V or a_stride below 1. */
kvx_status kvx_verify(const kvx_drafts *drafts, int32_t dtype, const void *logits, int64_t stride,
                      const void *draft, int64_t draft_stride, const float *uniforms,
                      const float *samples, int32_t *accepted, int32_t a_stride, int32_t *counts,
                      int32_t *next_tokens, void *workspace, uint64_t workspace_bytes,
                      void *hip_stream);

/* Bytes for kvx_verify with (with_draft) or without the draft's logits. */
kvx_status kvx_verify_workspace(const kvx_drafts *drafts, int32_t with_draft, uint64_t *bytes);

#ifdef __cplusplus
}
#endif
#endif /* KVX_SERVE_H */
