// kvx_attend: how a call is cut into workgroups, and the join of its splits.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "kvx_attend_dev.h"

namespace kvx {
namespace {

// ---- splits joined -------------------------------------------------------------
//
// The sums of a (token, query head)'s splits, each relative to its own reference,
// are brought to the largest and added, always in the same order.  A wave to
// each pair, or a workgroup's four where there are many splits; a split's sum is
// read 16 bytes a lane, as many splits at once as lanes allow.
template <bool kBf16, int kWaves>
__global__ void __launch_bounds__(256) kvx_join_kernel(const AttendArgs a, int lg_lanes)
{
    __shared__ __attribute__((aligned(16))) float s_acc[4][256];
    __shared__ float s_top[4], s_sum[4];
    const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) >> 6;
    const int64_t pairs = int64_t(a.b.total_tokens) * a.q_heads;
    const int64_t at = kWaves == 4 ? int64_t(blockIdx.x) : int64_t(blockIdx.x) * 4 + wave;
    if (at >= pairs) return;
    const int part = kWaves == 4 ? wave : 0;
    const int token = int(at / a.q_heads), head = int(at - int64_t(token) * a.q_heads);
    const int r = request_at(a.b.starts, a.c.num_requests, token);
    if (r < 0 || r >= a.c.num_requests) return;
    const Request rq = request_of(a.c, a.b, r);
    if (token - rq.first >= rq.n) return;
    const float2* const ml = reinterpret_cast<const float2*>(a.part_ml);
    // this wave's splits: [begin, end)
    const int begin = a.splits * part / kWaves, end = a.splits * (part + 1) / kWaves;
    float top = -INFINITY;
    for (int s = begin + lane; s < end; s += 64) top = fmaxf(top, ml[s * pairs + at].x);
    for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    if constexpr (kWaves == 4) {
        if (lane == 0) s_top[wave] = top;
        __syncthreads();
        top = fmaxf(fmaxf(s_top[0], s_top[1]), fmaxf(s_top[2], s_top[3]));
    }
    const int D = a.c.dim, lanes = 1 << lg_lanes, d = 4 * (lane & (lanes - 1)), step = 64 >> lg_lanes;
    float acc[4] = {}, total = 0.0f;
    for (int s0 = begin; s0 < end; s0 += 64) {
        const float2 v = s0 + lane < end ? ml[(s0 + lane) * pairs + at] : make_float2(-INFINITY, 0.0f);
        // a split that saw nothing left no sum: -1
        const float f = v.x == -INFINITY ? -1.0f : __builtin_amdgcn_exp2f(v.x - top);
        total += f < 0.0f ? 0.0f : v.y * f;
        const uint64_t some = __ballot(!(f < 0.0f));
        const int n = some ? 64 - __builtin_clzll(some) : 0;
        const float* const from = a.part_o + (int64_t(s0) * pairs + at) * D + (d < D ? d : 0);
        for (int s = 0; s < n; s += 4 * step) {
            float4 x[4];
            float w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int mine = s + k * step + (lane >> lg_lanes);
                const float weight = __shfl(f, mine & 63);   // by all lanes: each may hold another's
                w[k] = mine < n ? weight : -1.0f;
                x[k] = *reinterpret_cast<const float4*>(from + min(mine, n - 1) * pairs * D);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (!(w[k] < 0.0f))
                    acc[0] += weighted(x[k].x, w[k]), acc[1] += weighted(x[k].y, w[k]),
                        acc[2] += weighted(x[k].z, w[k]), acc[3] += weighted(x[k].w, w[k]);
            }
        }
    }
    for (int o = 32; o; o >>= 1) total += __shfl_xor(total, o);
    for (int o = lanes; o < 64; o <<= 1)
#pragma unroll
        for (int k = 0; k < 4; ++k) acc[k] += __shfl_xor(acc[k], o);
    if constexpr (kWaves == 4) {
        if (lane == 0) s_sum[wave] = total;
        if (lane < lanes) *reinterpret_cast<float4*>(&s_acc[wave][d]) = make_float4(acc[0], acc[1], acc[2], acc[3]);
        __syncthreads();
        if (wave != 0) return;
        total = (s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            acc[k] = (s_acc[0][d + k] + s_acc[1][d + k]) + (s_acc[2][d + k] + s_acc[3][d + k]);
    }
    const float inv = total == 0.0f ? 0.0f : 1.0f / total;
    if (lane < lanes && d < D)
        *reinterpret_cast<uint2*>(a.out + token * a.out_stride + int64_t(head) * D + d) =
            total == 0.0f ? make_uint2(0, 0) : make_uint2(pack2<kBf16>(acc[0] * inv, acc[1] * inv),
                                                          pack2<kBf16>(acc[2] * inv, acc[3] * inv));
    if (a.lse && lane == 0)
        a.lse[at] = total == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(total) - kShift<kBf16>) * kLn2;
}

// (split, token, query head) triples, in a multiple of 4
int64_t plan_pairs(const AttendArgs& a, const AttendPlan& p)
{
    return (int64_t(a.b.total_tokens) * a.q_heads * p.splits + 3) & ~int64_t(3);
}

// waves of a pair: a request of 120000 slots: 102 us in all, 110 with a wave a pair; 64 of
// 512..8192: 220, 223 with a workgroup a pair
int join_waves(int splits) { return splits > 32 ? 4 : 1; }

int64_t join_groups(int32_t tokens, int32_t q_heads, int waves)
{
    const int64_t pairs = int64_t(tokens) * q_heads;
    return waves == 4 ? pairs : (pairs + 3) / 4;
}

template <bool kBf16, int kWaves>
int join_as(const AttendArgs& a, void* stream)
{
    int lg_lanes = 0;
    while ((4 << lg_lanes) < a.c.dim) ++lg_lanes;
    return launch_kernel(kvx_join_kernel<kBf16, kWaves>, join_groups(a.b.total_tokens, a.q_heads, kWaves), 256, stream,
                         a, lg_lanes);
}

int join(const AttendArgs& a, bool bf, void* stream)
{
    if (join_waves(a.splits) == 4) return bf ? join_as<true, 4>(a, stream) : join_as<false, 4>(a, stream);
    return bf ? join_as<true, 1>(a, stream) : join_as<false, 1>(a, stream);
}

int rows(const AttendArgs& a, const AttendPlan& p, int dtype, int cache_dtype, void* stream)
{
    switch (cache_dtype) {
    case KVX_FP8_E4M3FN: return launch_rows<kCodesE4m3>(a, p, dtype, stream);
    case KVX_FP8_E5M2: return launch_rows<kCodesE5m2>(a, p, dtype, stream);
    default: return launch_rows<kCodes16>(a, p, dtype, stream);
    }
}

}  // namespace

int launch_attend(const AttendArgs& given, const AttendPlan& p, int dtype, int cache_dtype,
                  void* workspace, void* stream)
{
    const bool bf = dtype == KVX_BF16;
    AttendArgs a = given;
    a.chunk = p.chunk;
    a.splits = p.splits;
    a.part_ml = static_cast<float*>(workspace);
    a.part_o = a.part_ml + 2 * plan_pairs(a, p);
    const int err = p.few ? launch_few(a, p, dtype, cache_dtype, stream)
                          : rows(a, p, dtype, cache_dtype, stream);
    return err || p.splits == 1 ? err : join(a, bf, stream);
}

double attend_threads(const kvx_cache& c, const kvx_batch& b, int32_t q_heads, const AttendPlan& p)
{
    // the rows kernel has a wave to 32 rows
    const int threads = p.few ? 256 : 2 * p.tile_rows;
    const double first = double(c.num_requests) * c.num_kv_heads * p.splits * p.row_tiles * threads;
    return p.splits == 1 ? first
                         : std::max(first, double(join_groups(b.total_tokens, q_heads, join_waves(p.splits))) * 256);
}

AttendPlan attend_plan(const kvx_cache& c, const kvx_batch& b, int32_t q_heads)
{
    AttendPlan p = {};
    p.rows = int(std::min<int64_t>(int64_t(b.max_tokens) * (q_heads / c.num_kv_heads), INT32_MAX));
    const bool eight_bit = c.dtype == KVX_FP8_E4M3FN || c.dtype == KVX_FP8_E5M2;
    const int64_t heads = int64_t(c.num_requests) * c.num_kv_heads;
    const int64_t pieces = heads * ((b.max_context + 1023) / 1024);
    // 17 to 32 rows: the few-rows kernel's registers do not hold more than 128 elements; it cuts
    // the slots finer, which serves small calls (32 query heads on one KV head, one request of 8000
    // slots: 17 us, 39 with the other kernel; trees of 4..8 nodes over an fp8 cache of 2048..16384
    // slots: 128, 133), and where a 16-bit cache's slots fill the card in any case the other kernel
    // reads them faster (the same trees, 64 of them, bf16: 330 us, 362 with this one; at 512 pieces
    // both take 48).
    p.few = p.rows <= 16 || (p.rows <= 32 && c.head_dim <= 128 &&
                             (eight_bit || pieces < 512));
    p.tile_rows = p.few ? (p.rows <= 16 ? 16 : 32) : p.rows <= 64 ? 64 : 128;
    p.row_tiles = (p.rows + p.tile_rows - 1) / p.tile_rows;
    if (p.few) {
        p.chunk = 512;
    } else {
        // Rows fill the card by themselves from about 3 workgroups per two of a CU's places on
        // (chunks of 1024..2048 tokens: 810 us in one split, 1043 in splits of 2048 slots, whose
        // sums have to be written and joined); fewer are split, the bounds counting requests
        // shorter than the longest as idle workgroups (trees of 16..64 nodes over 2048..16384
        // slots: 687 us in one split, 403 with 2048 slots, 392 with 1024, 433 with 512).
        const int64_t groups = heads * p.row_tiles;
        const int64_t want = groups >= 768 ? 1 : (4096 + groups - 1) / groups;
        // Few workgroups in all are cut down to 256 slots, until there is one to a CU (a tree over
        // 6000 slots, 8 KV heads: 24 us, 48 with 1024 slots at least; one head, 120000 slots: 39,
        // 54); beyond that the join eats what is won (16 trees over 900 slots: 54 us with two to a
        // CU, 47 with one).
        const int64_t least = std::min<int64_t>(1024, std::max<int64_t>(256, groups * b.max_context / 256));
        p.chunk = int((std::max(least, (b.max_context + want - 1) / want) + 63) & ~int64_t(63));
    }
    p.splits = (b.max_context + p.chunk - 1) / p.chunk;
    return p;
}

uint64_t attend_workspace(const kvx_cache& c, const kvx_batch& b, int32_t q_heads)
{
    const AttendPlan p = attend_plan(c, b, q_heads);
    if (p.splits == 1) return 0;
    const uint64_t pairs = (uint64_t(b.total_tokens) * q_heads * p.splits + 3) & ~uint64_t(3);
    return pairs * (2 + uint64_t(c.head_dim)) * 4;
}

}  // namespace kvx
