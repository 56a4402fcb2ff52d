/*
 * kvx_ops.h -- C ABI of the operators that a decode engine runs on its paged
 * cache, beside the conversions of kvx.h that fill it.
 *
 *   kvx_append  rotary positions on the new tokens' queries and keys; keys and
 *               values written into the cache
 *   kvx_attend  attention of the new tokens (one, a drafted tree or a chain)
 *               over the cache
 *   kvx_weigh   the attention weight of every cache slot, accumulated
 *   kvx_evict   the slots of the largest weights kept, moved up in place
 *   kvx_commit  the accepted path of a drafted tree moved to the front
 *
 * The cache is the one that kvx_unpack and kvx_repack write:
 * [layer][k/v][num_blocks][block_size][Hd][D] and, for 8-bit codes, fp32 scales
 * [layer][k/v][num_blocks][block_size][Hd]; or one of 4 bits, which kvx_append fills
 * (KVX_FP4_E2M1).  Slot j of request r is slot
 * j % block_size of page block_table[r * bt_stride + j / block_size].  A page id
 * outside [0, num_blocks) names no page: its slots are not seen by attention,
 * weigh nothing, and are neither moved nor written.  Requests may name the same page
 * where they only read it; slots that kvx_append writes, or that kvx_evict and
 * kvx_commit move, lie in pages of one request alone.
 *
 * A batch holds the new tokens of the requests, request r's at tokens
 * token_starts[r] .. token_starts[r + 1] - 1 of the flat token axis, n_r of
 * them.  contexts[r] = C_r slots of its row are in use before them; they take
 * slots C_r .. C_r + n_r - 1.  Lengths, tables, positions and trees are read on
 * the device when the kernels run, so a recorded graph follows them; the host
 * gives bounds only (total_tokens, max_tokens, max_context).  Device values
 * outside those bounds are cut to them: no access leaves the buffers that the
 * bounds describe.
 *
 * Ownership, streams and errors are those of kvx.h: every buffer is the
 * caller's, calls only launch kernels on the given hipStream_t (void*, NULL =
 * default stream) and may be recorded into a HIP graph; a kvx_status comes back
 * and kvx_last_error() has its message.  A call with nothing to do returns
 * KVX_OK without inspecting its data pointers; one that would need 2^32 threads or
 * more in a launch (2^24 workgroups of 256) returns KVX_EUNSUPPORTED before the
 * first.  Results are the same in every
 * run: no sum depends on the order in which workgroups end.
 */
#ifndef KVX_OPS_H
#define KVX_OPS_H

#include "kvx.h"

#ifdef __cplusplus
extern "C" {
#endif

#define KVX_OPS_VERSION 1

/* A cache's element type beside those of kvx_dtype: e2m1 codes (0, 0.5, 1, 1.5, 2, 3, 4,
 * 6 and their negatives; the sign is bit 3), two a byte, the element of the even
 * number in the lower bits, [layer][k/v][num_blocks][block_size][Hd][D / 2], and a
 * scale byte b for every 32 elements of a row,
 * [layer][k/v][num_blocks][block_size][Hd][D / 32]: an element is its code's value times
 * 2^(b - 127), and NaN where b is above 252.  kvx_append takes the smallest scale with
 * |x| <= 7 scale in the group, so that no element is off by more than half a step of its
 * size, cut to 2^-126 .. 2^125, and divides, rounds to nearest even and cuts at 6; a group
 * with an element that is not finite becomes NaN. */
#define KVX_FP4_E2M1 5

int32_t kvx_ops_version(void);

/* A decode rank's paged cache and the block table of the requests at hand. */
typedef struct {
    int32_t num_layers;
    int32_t num_kv_heads;       /* Hd: KV heads of this rank */
    int32_t head_dim;           /* D: a multiple of 8 (16-bit), 16 (8-bit) or 32 (4-bit), at most 256 */
    int32_t dtype;              /* kvx_dtype of the cache, or KVX_FP4_E2M1 */
    int32_t block_size;         /* slots per page */
    int32_t num_requests;       /* rows of the block table */
    int32_t bt_stride;          /* entries per row */
    int32_t reserved;
    int64_t num_blocks;         /* pages per (layer, k/v) plane */
    void *cache;                /* device, 16-byte aligned */
    float *scales;              /* device, non-NULL if and only if dtype is 8-bit or 4-bit (the
                                 * scale bytes then, cast, 16-byte aligned) */
    const int32_t *block_table; /* device [num_requests][bt_stride] */
} kvx_cache;

/* The new tokens of those requests. */
typedef struct {
    int32_t total_tokens;       /* N: tokens of the flat axis, >= 0 */
    int32_t max_tokens;         /* bound of n_r, 1 .. 65536 */
    int32_t max_context;        /* bound of C_r + n_r, 1 .. bt_stride * block_size */
    int32_t tree_stride;        /* 64-bit words per token of `tree`; 64 * tree_stride >= max_tokens */
    const int32_t *token_starts;/* device [num_requests + 1], non-decreasing, within 0 .. N */
    const int32_t *contexts;    /* device [num_requests] */
    const int32_t *positions;   /* device [N] or NULL: the position of each new token that a bias or
                                 * a window goes by, within +-2^30; NULL: C_r + i for token i of
                                 * request r.  Slot j < C_r has position j. */
    const uint64_t *tree;       /* device [N][tree_stride] or NULL: bit j of token i's words says
                                 * whether it sees new token j of its request (itself included).
                                 * NULL: a chain, token i sees tokens 0 .. i. */
} kvx_batch;

/* How scores are formed from the products s = q . k:
 *   x = scale * s;  softcap > 0: x = softcap * tanh(x / softcap);
 *   slopes: x -= slopes[query head] * |position of the token - position of the slot|.
 * Slot j is visible to token i of request r when j < prefix[r], or when
 *   (j < C_r, or the tree says so) and, for window > 0,
 *   position of the token - position of the slot < window.
 * A slot in use has its own number as its position, also after kvx_evict has moved
 * another token's row there (each head its own): over an evicted request a bias and a
 * window go by slots, and positions counted in slots (kvx_batch.positions NULL)
 * belong to them.  What lies further back than the tokens between is then nearer. */
typedef struct {
    float scale;
    float softcap;              /* 0: none */
    int32_t window;             /* 0: none */
    int32_t reserved;
    const float *slopes;        /* device [q_heads] or NULL */
    const int32_t *prefix;      /* device [num_requests] or NULL: slots visible to every token */
} kvx_scores;

/* Rotary positions.  `pairs` pairs of elements of every head turn: pair i is
 * (i, i + pairs) or, interleaved, (2i, 2i + 1); elements from 2 * pairs on stay.
 * Pair i belongs to the axis in whose section it lies (sections are
 * consecutive and sum to `pairs`) and turns by the angle
 * position[axis][token] * inv_freq[i], that product rounded to fp32. */
typedef struct {
    int32_t pairs;              /* 0 .. D / 2 */
    int32_t interleaved;
    int32_t num_axes;           /* 1 .. 4 */
    int32_t sections[4];
    int32_t reserved;
    const float *inv_freq;      /* device [pairs] */
    const int32_t *positions;   /* device [num_axes][N] */
} kvx_rope;

/* Turns q and k and writes the new tokens' keys and values into layer `layer`.
 *   dtype:   KVX_FP16 or KVX_BF16, the type of q, k, v and q_out.
 *   q, k, v: device; token t's heads are [heads][D] at t * stride elements
 *            (q_heads heads for q, Hd for k and v; strides are multiples of 8,
 *            pointers 16-byte aligned, so slices of a fused projection serve).
 *   q_out:   device, likewise; may be q itself.  q and q_out both NULL with
 *            q_heads 0: keys and values only.
 * Values are turned in fp32 and rounded once: q to dtype, k and v to the
 * cache's type (to nearest even; an 8-bit cache takes the casts of kvx.h, its
 * scale from the fp32 row, a 4-bit one KVX_FP4_E2M1's).  Tokens whose slot has no page write no row.  A 16-bit
 * cache may have the other 16-bit type than k and v; kvx_attend and kvx_weigh then
 * take queries of the cache's type.
 * KVX_EINVAL: NULL or misaligned pointers, sizes out of the ranges above, layer
 * outside the cache.  KVX_EUNSUPPORTED: head_dim above 256. */
kvx_status kvx_append(const kvx_cache *cache, const kvx_batch *batch, const kvx_rope *rope,
                      int32_t layer, int32_t dtype, int32_t q_heads, const void *q,
                      int64_t q_stride, const void *k, int64_t k_stride, const void *v,
                      int64_t v_stride, void *q_out, int64_t q_out_stride, void *hip_stream);

/* Attention of the batch's tokens over layer `layer`; the new tokens' rows are
 * in the cache already.  Query head h reads KV head h / (q_heads / Hd).
 *   q, out:    dtype, layout and strides as above.
 *   lse:       device fp32 [N][q_heads] or NULL: log of the sum of exp(x).
 *   workspace: device, >= kvx_attend_workspace bytes, 16-byte aligned; NULL if
 *              that is 0.  Its contents need not be kept between calls; calls (and graphs)
 *              that may run at the same time need one each.
 * A token that sees no slot, or whose scores are all -infinity, gives zeros and an
 * lse of -infinity; a NaN among its scores (from q or from a key that it sees)
 * gives NaN in both.  An infinite value in a slot that it sees makes that element of
 * the result infinite however small the slot's weight is, opposite infinities or a
 * NaN make it NaN (a score of -infinity leaves open whether its slot's values
 * count).  What lies in slots that a token does not see (infinities and NaN too) has
 * no part in its result.  Scores, softmax statistics and sums are fp32.  For the
 * product with V weights are rounded to 16 bits, with max_tokens * q_heads / Hd <= 16
 * to twice as many; over a 4-bit cache both products are of bf16, fp16 queries and
 * their weights in two such terms; the output is rounded once to dtype.  A 16-bit cache must have
 * the type of q (KVX_EUNSUPPORTED otherwise); q_heads is a multiple of Hd with at
 * most 1024 query heads per KV head. */
kvx_status kvx_attend(const kvx_cache *cache, const kvx_batch *batch, const kvx_scores *scores,
                      int32_t layer, int32_t dtype, int32_t q_heads, const void *q,
                      int64_t q_stride, void *out, int64_t out_stride, float *lse,
                      void *workspace, uint64_t workspace_bytes, void *hip_stream);

kvx_status kvx_attend_workspace(const kvx_cache *cache, const kvx_batch *batch, int32_t q_heads,
                                uint64_t *bytes);

/* The attention weight of the cache's slots: for KV head g and slot j of
 * request r, the sum over the batch's tokens and the query heads of g of
 * exp(x - lse), with x and visibility as in kvx_attend and lse what that call
 * gave (a token with lse -infinity weighs nothing, one with lse NaN makes the sums
 * of the slots that it sees NaN).
 *   weights: device fp32 [num_requests][Hd][w_stride], w_stride >= max_context:
 *            slots j < C_r have the sum added, the new tokens' slots are set to
 *            it, others are not touched.
 * KVX_EUNSUPPORTED: a 4-bit cache, and as kvx_attend. */
kvx_status kvx_weigh(const kvx_cache *cache, const kvx_batch *batch, const kvx_scores *scores,
                     int32_t layer, int32_t dtype, int32_t q_heads, const void *q,
                     int64_t q_stride, const float *lse, float *weights, int64_t w_stride,
                     void *hip_stream);

/* Eviction in layers layer0 .. layer0 + num_layers - 1.  Request r has
 * lens[r] = T slots in use (cut to max_len); with T <= budget all stay,
 * otherwise `budget` of them: the first `sink`, the last `recent`, and of those
 * between the ones of the largest weight (ties: the lowest slot; -0 equals 0;
 * NaN counts above infinity), chosen for every layer and KV head.  Kept rows
 * move up to slots 0 .. budget - 1 in their order, keys, values and scales.
 *   weights:     device fp32 [num_layers][num_requests][Hd][w_stride],
 *                w_stride >= max_len.
 *   weights_out: device, the same layout: the kept slots' weights at 0 .. keep
 *                - 1, nothing else written.  May be `weights`.
 *   kept:        device int32 [num_layers][num_requests][Hd][budget]: the kept
 *                slots in ascending order, then -1.
 *   new_lens:    device int32 [num_requests]: min(T, budget); another buffer than
 *                lens.
 * sink + recent <= budget, budget >= 1, max_len <= bt_stride * block_size. */
kvx_status kvx_evict(const kvx_cache *cache, int32_t layer0, int32_t num_layers,
                     const int32_t *lens, int32_t max_len, int32_t budget, int32_t sink,
                     int32_t recent, const float *weights, float *weights_out, int64_t w_stride,
                     int32_t *kept, int32_t *new_lens, void *hip_stream);

/* After a drafted tree has been verified: in layers layer0 .. layer0 +
 * num_layers - 1, slot contexts[r] + i takes the row of slot contexts[r] +
 * accepted[r * a_stride + i], for i < counts[r] (cut to a_stride), keys, values
 * and scales.  accepted[r] ascends strictly from 0 or more (a path of a tree
 * whose nodes come after their parents); an entry that is not above the one
 * before it, or whose slot is outside the block-table row, ends the path there.
 *   new_lens: device int32 [num_requests]: contexts[r] + the length of the path;
 *             another buffer than contexts. */
kvx_status kvx_commit(const kvx_cache *cache, int32_t layer0, int32_t num_layers,
                      const int32_t *contexts, const int32_t *accepted, int32_t a_stride,
                      const int32_t *counts, int32_t *new_lens, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* KVX_OPS_H */
