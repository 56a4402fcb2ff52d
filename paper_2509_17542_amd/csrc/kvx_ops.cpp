// Host side of the decode operators (kvx_ops.h, kvx_fetch of kvx_serve.h): argument checks and
// launches.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cmath>

#include "kvx_host.h"
#include "kvx_ops_internal.h"

namespace {

using kvx::fail;

bool is_fp8(int dt) { return dt == KVX_FP8_E4M3FN || dt == KVX_FP8_E5M2; }

bool is_fp4(int dt) { return dt == KVX_FP4_E2M1; }

bool is_16bit(int dt) { return dt == KVX_FP16 || dt == KVX_BF16; }

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// slots of one request
constexpr int32_t kMaxSlots = 1 << 30;

int64_t row_slots(const kvx_cache& c) { return int64_t(c.bt_stride) * c.block_size; }

kvx_status check_shape(const kvx_cache* c)
{
    if (!c) return fail(KVX_EINVAL, "NULL cache");
    if (c->num_layers < 1 || c->num_kv_heads < 1 || c->head_dim < 1 || c->block_size < 1 ||
        c->num_blocks < 1)
        return fail(KVX_EINVAL, "a cache's layers, heads, head_dim, block_size and num_blocks must be >= 1");
    if (!is_fp8(c->dtype) && !is_16bit(c->dtype) && !is_fp4(c->dtype))
        return fail(KVX_EINVAL, "unknown cache dtype %d", c->dtype);
    if (c->num_requests < 0 || c->bt_stride < 0)
        return fail(KVX_EINVAL, "num_requests and bt_stride must be >= 0");
    if (is_fp4(c->dtype) && c->head_dim % 32)
        return fail(KVX_EINVAL, "head_dim %d: rows of a 4-bit cache must be whole groups of 32", c->head_dim);
    if (c->head_dim % (is_fp8(c->dtype) ? 16 : 8))
        return fail(KVX_EINVAL, "head_dim %d: rows must be whole 16-byte vectors", c->head_dim);
    if (c->head_dim > 256) return fail(KVX_EUNSUPPORTED, "head_dim %d above 256", c->head_dim);
    if (c->num_kv_heads > kvx::kMaxHeadsPerRank)
        return fail(KVX_EUNSUPPORTED, "more than %d heads per decode rank", kvx::kMaxHeadsPerRank);
    const double slots = double(c->num_layers) * 2 * double(c->num_blocks) * c->block_size *
                         c->num_kv_heads;
    if (slots * c->head_dim * 2 >= 0x1p62) return fail(KVX_EUNSUPPORTED, "cache above 2^62 bytes");
    return KVX_OK;
}

// Buffers of a cache that kernels will touch.
kvx_status check_buffers(const kvx_cache& c)
{
    if (!c.cache || !c.block_table) return fail(KVX_EINVAL, "NULL cache or block table");
    if (!aligned16(c.cache)) return fail(KVX_EINVAL, "the cache must be 16-byte aligned");
    if ((is_fp8(c.dtype) || is_fp4(c.dtype)) != (c.scales != nullptr))
        return fail(KVX_EINVAL, "scales must be given exactly for an 8-bit or a 4-bit cache");
    if (is_fp4(c.dtype) && !aligned16(c.scales))
        return fail(KVX_EINVAL, "the scale bytes must be 16-byte aligned");
    return KVX_OK;
}

kvx_status check_layers(const kvx_cache& c, int64_t layer0, int64_t n)
{
    if (layer0 < 0 || n < 0 || layer0 + n > c.num_layers)
        return fail(KVX_EINVAL, "layers [%lld, %lld) outside the cache's %d", (long long)layer0,
                    (long long)(layer0 + n), c.num_layers);
    return KVX_OK;
}

kvx_status check_batch(const kvx_cache& c, const kvx_batch* b)
{
    if (!b) return fail(KVX_EINVAL, "NULL batch");
    if (b->total_tokens < 0) return fail(KVX_EINVAL, "total_tokens must be >= 0");
    if (b->total_tokens == 0 || c.num_requests == 0) return KVX_OK;
    if (b->max_tokens < 1 || b->max_tokens > 65536)
        return fail(KVX_EINVAL, "max_tokens %d outside [1, 65536]", b->max_tokens);
    if (b->max_context < 1 || b->max_context > row_slots(c))
        return fail(KVX_EINVAL, "max_context %d outside [1, %lld], the slots of a block-table row",
                    b->max_context, (long long)row_slots(c));
    if (b->max_context > kMaxSlots)
        return fail(KVX_EUNSUPPORTED, "max_context %d above 2^30", b->max_context);
    if (!b->token_starts || !b->contexts) return fail(KVX_EINVAL, "NULL token_starts or contexts");
    if (b->tree && (b->tree_stride < 1 || int64_t(b->tree_stride) * 64 < b->max_tokens))
        return fail(KVX_EINVAL, "tree_stride %d: %d tokens need a bit each", b->tree_stride,
                    b->max_tokens);
    return KVX_OK;
}

kvx_status check_rows(const char* what, const void* p, int64_t stride, int64_t width)
{
    if (!p) return fail(KVX_EINVAL, "NULL %s", what);
    if (!aligned16(p) || stride % 8)
        return fail(KVX_EINVAL, "%s: tokens must start at 16-byte boundaries", what);
    if (stride < width)
        return fail(KVX_EINVAL, "%s: stride %lld below the %lld elements of a token", what,
                    (long long)stride, (long long)width);
    return KVX_OK;
}

kvx::CacheArgs cache_args(const kvx_cache& c, int layer0)
{
    kvx::CacheArgs a = {};
    const bool four = is_fp4(c.dtype);
    a.row_bytes = four ? c.head_dim / 2 : c.head_dim * (is_fp8(c.dtype) ? 1 : 2);
    a.row_groups = four ? c.head_dim / 32 : 0;
    a.plane_scales = c.num_blocks * c.block_size * c.num_kv_heads;
    a.plane_bytes = a.plane_scales * a.row_bytes;
    a.base = static_cast<char*>(c.cache) + 2 * int64_t(layer0) * a.plane_bytes;
    if (four)
        a.groups = reinterpret_cast<uint8_t*>(c.scales) + 2 * int64_t(layer0) * a.plane_scales * a.row_groups;
    else if (c.scales)
        a.scales = c.scales + 2 * int64_t(layer0) * a.plane_scales;
    a.table = c.block_table;
    a.num_blocks = c.num_blocks;
    a.bt_stride = c.bt_stride;
    a.block_size = c.block_size;
    a.hd = c.num_kv_heads;
    a.dim = c.head_dim;
    a.row_slots = int32_t(std::min<int64_t>(row_slots(c), kMaxSlots));
    a.num_requests = c.num_requests;
    a.div_bs = kvx::make_fastdiv(uint32_t(c.block_size));
    return a;
}

kvx::BatchArgs batch_args(const kvx_batch& b)
{
    kvx::BatchArgs a = {};
    a.starts = b.token_starts;
    a.contexts = b.contexts;
    a.positions = b.positions;
    a.tree = b.tree;
    a.tree_stride = b.tree_stride;
    a.total_tokens = b.total_tokens;
    a.max_tokens = b.max_tokens;
    a.max_context = b.max_context;
    return a;
}

kvx_status launched(int err)
{
    if (err == int(hipSuccess)) return KVX_OK;
    return fail(KVX_EDEVICE, "kernel launch failed: %s", hipGetErrorString(hipError_t(err)));
}

kvx_status need_device()
{
    int dev = -1;
    const hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return fail(KVX_EDEVICE, "no HIP device: %s", hipGetErrorString(e));
    return KVX_OK;
}

// threads of a call's largest launch
kvx_status check_threads(double threads)
{
    if (threads >= 0x1p32) return fail(KVX_EUNSUPPORTED, "%.0f threads in a launch: 2^32 or more", threads);
    return KVX_OK;
}

#define KVX_TRY(call)                              \
    do {                                           \
        const kvx_status status_ = (call);         \
        if (status_ != KVX_OK) return status_;     \
    } while (0)

// What kvx_attend and kvx_weigh check alike; *idle: there is nothing to do.
kvx_status check_scores(const kvx_cache* c, const kvx_batch* b, const kvx_scores* s, int32_t layer,
                        int32_t dtype, int32_t q_heads, bool* idle)
{
    KVX_TRY(check_shape(c));
    KVX_TRY(check_batch(*c, b));
    KVX_TRY(check_layers(*c, layer, 1));
    if (!s) return fail(KVX_EINVAL, "NULL scores");
    if (!std::isfinite(s->scale)) return fail(KVX_EINVAL, "scale must be finite");
    if (!(s->softcap >= 0.0f) || !std::isfinite(s->softcap))
        return fail(KVX_EINVAL, "softcap must be finite and >= 0");
    if (s->window < 0) return fail(KVX_EINVAL, "window must be >= 0");
    if (!is_16bit(dtype)) return fail(KVX_EINVAL, "q must be KVX_FP16 or KVX_BF16, not %d", dtype);
    if (is_16bit(c->dtype) && c->dtype != dtype)
        return fail(KVX_EUNSUPPORTED, "a 16-bit cache must have the type of q");
    if (q_heads < 1 || q_heads % c->num_kv_heads)
        return fail(KVX_EINVAL, "q_heads %d is not a multiple of %d KV heads", q_heads,
                    c->num_kv_heads);
    if (q_heads / c->num_kv_heads > 1024)
        return fail(KVX_EUNSUPPORTED, "more than 1024 query heads per KV head");
    *idle = b->total_tokens == 0 || c->num_requests == 0;
    return KVX_OK;
}

kvx::AttendArgs attend_args(const kvx_cache& c, const kvx_batch& b, const kvx_scores& s,
                            int32_t layer, int32_t q_heads)
{
    kvx::AttendArgs a = {};
    a.c = cache_args(c, layer);
    a.b = batch_args(b);
    a.slopes = s.slopes;
    a.prefix = s.prefix;
    a.scale = s.scale;
    a.softcap = s.softcap;
    a.window = s.window;
    a.q_heads = q_heads;
    a.group = q_heads / c.num_kv_heads;
    a.div_group = kvx::make_fastdiv(uint32_t(a.group));
    return a;
}

}  // namespace

extern "C" int32_t kvx_ops_version(void) { return KVX_OPS_VERSION; }

extern "C" kvx_status kvx_append(const kvx_cache* c, const kvx_batch* b, const kvx_rope* rope,
                                 int32_t layer, int32_t dtype, int32_t q_heads, const void* q,
                                 int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                                 int64_t v_stride, void* q_out, int64_t q_out_stride, void* stream)
{
    KVX_TRY(check_shape(c));
    KVX_TRY(check_batch(*c, b));
    KVX_TRY(check_layers(*c, layer, 1));
    if (!rope) return fail(KVX_EINVAL, "NULL rope");
    if (rope->pairs < 0 || 2 * int64_t(rope->pairs) > c->head_dim)
        return fail(KVX_EINVAL, "%d pairs do not fit head_dim %d", rope->pairs, c->head_dim);
    if (rope->num_axes < 1 || rope->num_axes > 4)
        return fail(KVX_EINVAL, "num_axes %d outside [1, 4]", rope->num_axes);
    int64_t sum = 0;
    for (int i = 0; i < rope->num_axes; ++i) {
        if (rope->sections[i] < 0) return fail(KVX_EINVAL, "sections[%d] < 0", i);
        sum += rope->sections[i];
    }
    if (sum != rope->pairs)
        return fail(KVX_EINVAL, "sections sum to %lld, not to the %d pairs", (long long)sum, rope->pairs);
    if (!is_16bit(dtype)) return fail(KVX_EINVAL, "q, k, v must be KVX_FP16 or KVX_BF16, not %d", dtype);
    if (q_heads < 0 || q_heads > 65536) return fail(KVX_EINVAL, "q_heads %d outside [0, 65536]", q_heads);
    if (b->total_tokens == 0 || c->num_requests == 0) return KVX_OK;
    KVX_TRY(check_buffers(*c));
    if (rope->pairs > 0 && (!rope->inv_freq || !rope->positions))
        return fail(KVX_EINVAL, "NULL inv_freq or positions");
    const int64_t kv_width = int64_t(c->num_kv_heads) * c->head_dim;
    if (q_heads > 0) {
        KVX_TRY(check_rows("q", q, q_stride, int64_t(q_heads) * c->head_dim));
        KVX_TRY(check_rows("q_out", q_out, q_out_stride, int64_t(q_heads) * c->head_dim));
    }
    KVX_TRY(check_rows("k", k, k_stride, kv_width));
    KVX_TRY(check_rows("v", v, v_stride, kv_width));
    KVX_TRY(check_threads(kvx::append_threads(b->total_tokens)));
    KVX_TRY(need_device());
    kvx::AppendArgs a = {};
    a.c = cache_args(*c, layer);
    a.b = batch_args(*b);
    a.q = static_cast<const uint16_t*>(q);
    a.k = static_cast<const uint16_t*>(k);
    a.v = static_cast<const uint16_t*>(v);
    a.q_out = static_cast<uint16_t*>(q_out);
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.q_out_stride = q_out_stride;
    a.inv_freq = rope->inv_freq;
    a.positions = rope->positions;
    a.q_heads = q_heads;
    a.pairs = rope->pairs;
    a.interleaved = rope->interleaved != 0;
    for (int i = 0, end = 0; i < 4; ++i) {
        end = i < rope->num_axes ? end + rope->sections[i] : rope->pairs;
        a.sec_end[i] = end;
    }
    while ((8 << a.lg_row) < c->head_dim) ++a.lg_row;
    return launched(kvx::launch_append(a, dtype, c->dtype, stream));
}

extern "C" int32_t kvx_serve_version(void) { return KVX_SERVE_VERSION; }

extern "C" kvx_status kvx_fetch(const kvx_cache* c, const kvx_batch* b, int32_t layer, int32_t dtype,
                                void* k, int64_t k_stride, void* v, int64_t v_stride, void* stream)
{
    KVX_TRY(check_shape(c));
    KVX_TRY(check_batch(*c, b));
    KVX_TRY(check_layers(*c, layer, 1));
    if (!is_16bit(dtype)) return fail(KVX_EINVAL, "k and v must be KVX_FP16 or KVX_BF16, not %d", dtype);
    if (b->total_tokens == 0 || c->num_requests == 0) return KVX_OK;
    KVX_TRY(check_buffers(*c));
    const int64_t width = int64_t(c->num_kv_heads) * c->head_dim;
    KVX_TRY(check_rows("k", k, k_stride, width));
    KVX_TRY(check_rows("v", v, v_stride, width));
    KVX_TRY(check_threads(kvx::fetch_threads(b->total_tokens)));
    KVX_TRY(need_device());
    kvx::FetchArgs a = {};
    a.c = cache_args(*c, layer);
    a.b = batch_args(*b);
    a.k = static_cast<uint16_t*>(k);
    a.v = static_cast<uint16_t*>(v);
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    return launched(kvx::launch_fetch(a, dtype, c->dtype, stream));
}

extern "C" kvx_status kvx_attend_workspace(const kvx_cache* c, const kvx_batch* b, int32_t q_heads,
                                           uint64_t* bytes)
{
    if (!bytes) return fail(KVX_EINVAL, "NULL bytes");
    KVX_TRY(check_shape(c));
    KVX_TRY(check_batch(*c, b));
    if (q_heads < 1 || q_heads % c->num_kv_heads)
        return fail(KVX_EINVAL, "q_heads %d is not a multiple of %d KV heads", q_heads,
                    c->num_kv_heads);
    *bytes = b->total_tokens == 0 || c->num_requests == 0 ? 0 : kvx::attend_workspace(*c, *b, q_heads);
    return KVX_OK;
}

extern "C" kvx_status kvx_attend(const kvx_cache* c, const kvx_batch* b, const kvx_scores* s,
                                 int32_t layer, int32_t dtype, int32_t q_heads, const void* q,
                                 int64_t q_stride, void* out, int64_t out_stride, float* lse,
                                 void* workspace, uint64_t workspace_bytes, void* stream)
{
    bool idle = false;
    KVX_TRY(check_scores(c, b, s, layer, dtype, q_heads, &idle));
    if (idle) return KVX_OK;
    KVX_TRY(check_buffers(*c));
    KVX_TRY(check_rows("q", q, q_stride, int64_t(q_heads) * c->head_dim));
    KVX_TRY(check_rows("out", out, out_stride, int64_t(q_heads) * c->head_dim));
    const uint64_t need = kvx::attend_workspace(*c, *b, q_heads);
    if (need && (!workspace || workspace_bytes < need || !aligned16(workspace)))
        return fail(KVX_EINVAL, "a 16-byte aligned workspace of %llu bytes is needed, %llu are given",
                    (unsigned long long)need, (unsigned long long)(workspace ? workspace_bytes : 0));
    const kvx::AttendPlan plan = kvx::attend_plan(*c, *b, q_heads);
    KVX_TRY(check_threads(kvx::attend_threads(*c, *b, q_heads, plan)));
    KVX_TRY(need_device());
    kvx::AttendArgs a = attend_args(*c, *b, *s, layer, q_heads);
    a.q = static_cast<const uint16_t*>(q);
    a.out = static_cast<uint16_t*>(out);
    a.lse = lse;
    a.q_stride = q_stride;
    a.out_stride = out_stride;
    return launched(kvx::launch_attend(a, plan, dtype, c->dtype, workspace, stream));
}

extern "C" kvx_status kvx_weigh(const kvx_cache* c, const kvx_batch* b, const kvx_scores* s,
                                int32_t layer, int32_t dtype, int32_t q_heads, const void* q,
                                int64_t q_stride, const float* lse, float* weights,
                                int64_t w_stride, void* stream)
{
    bool idle = false;
    KVX_TRY(check_scores(c, b, s, layer, dtype, q_heads, &idle));
    if (idle) return KVX_OK;
    KVX_TRY(check_buffers(*c));
    KVX_TRY(check_rows("q", q, q_stride, int64_t(q_heads) * c->head_dim));
    if (!lse || !weights) return fail(KVX_EINVAL, "NULL lse or weights");
    if (w_stride < b->max_context)
        return fail(KVX_EINVAL, "w_stride %lld below max_context %d", (long long)w_stride, b->max_context);
    if (is_fp4(c->dtype)) return fail(KVX_EUNSUPPORTED, "kvx_weigh over a 4-bit cache");
    KVX_TRY(check_threads(kvx::weigh_threads(*c, *b, q_heads)));
    KVX_TRY(need_device());
    kvx::AttendArgs a = attend_args(*c, *b, *s, layer, q_heads);
    a.q = static_cast<const uint16_t*>(q);
    a.q_stride = q_stride;
    a.lse = const_cast<float*>(lse);
    a.weights = weights;
    a.w_stride = w_stride;
    return launched(kvx::launch_weigh(a, dtype, c->dtype, stream));
}

extern "C" kvx_status kvx_evict(const kvx_cache* c, int32_t layer0, int32_t num_layers,
                                const int32_t* lens, int32_t max_len, int32_t budget, int32_t sink,
                                int32_t recent, const float* weights, float* weights_out,
                                int64_t w_stride, int32_t* kept, int32_t* new_lens, void* stream)
{
    KVX_TRY(check_shape(c));
    KVX_TRY(check_layers(*c, layer0, num_layers));
    if (max_len < 0 || max_len > row_slots(*c))
        return fail(KVX_EINVAL, "max_len %d outside [0, %lld], the slots of a block-table row", max_len,
                    (long long)row_slots(*c));
    if (max_len > kMaxSlots) return fail(KVX_EUNSUPPORTED, "max_len %d above 2^30", max_len);
    if (budget < 1 || sink < 0 || recent < 0 || int64_t(sink) + recent > budget)
        return fail(KVX_EINVAL, "budget %d must be >= 1 and hold sink %d + recent %d", budget, sink, recent);
    if (w_stride < max_len)
        return fail(KVX_EINVAL, "w_stride %lld below max_len %d", (long long)w_stride, max_len);
    if (num_layers == 0 || c->num_requests == 0) return KVX_OK;
    KVX_TRY(check_buffers(*c));
    if (!lens || !weights || !weights_out || !kept || !new_lens)
        return fail(KVX_EINVAL, "NULL lens, weights, weights_out, kept or new_lens");
    if (new_lens == lens) return fail(KVX_EINVAL, "new_lens must be another buffer than lens");
    kvx::EvictArgs a = {};
    a.c = cache_args(*c, layer0);
    KVX_TRY(check_threads(kvx::evict_threads(a.c, num_layers, max_len)));
    KVX_TRY(need_device());
    a.lens = lens;
    a.weights = weights;
    a.weights_out = weights_out;
    a.kept = kept;
    a.new_lens = new_lens;
    a.w_stride = w_stride;
    a.max_len = max_len;
    a.budget = budget;
    a.sink = sink;
    a.recent = recent;
    return launched(kvx::launch_evict(a, num_layers, stream));
}

extern "C" kvx_status kvx_commit(const kvx_cache* c, int32_t layer0, int32_t num_layers,
                                 const int32_t* contexts, const int32_t* accepted, int32_t a_stride,
                                 const int32_t* counts, int32_t* new_lens, void* stream)
{
    KVX_TRY(check_shape(c));
    KVX_TRY(check_layers(*c, layer0, num_layers));
    if (a_stride < 0) return fail(KVX_EINVAL, "a_stride must be >= 0");
    if (c->num_requests == 0) return KVX_OK;
    if (!contexts || !counts || !new_lens || (a_stride > 0 && !accepted))
        return fail(KVX_EINVAL, "NULL contexts, accepted, counts or new_lens");
    if (new_lens == contexts) return fail(KVX_EINVAL, "new_lens must be another buffer than contexts");
    if (num_layers > 0) KVX_TRY(check_buffers(*c));
    kvx::CommitArgs a = {};
    a.c = cache_args(*c, layer0);
    KVX_TRY(check_threads(kvx::commit_threads(a.c, num_layers)));
    KVX_TRY(need_device());
    a.contexts = contexts;
    a.accepted = accepted;
    a.counts = counts;
    a.new_lens = new_lens;
    a.a_stride = a_stride;
    a.num_layers = num_layers;
    return launched(kvx::launch_commit(a, stream));
}
