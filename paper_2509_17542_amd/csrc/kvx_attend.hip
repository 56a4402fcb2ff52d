// gfx950 kernels of attention over the paged cache (kvx_attend) and of the
// slots' accumulated weights (kvx_weigh).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "kvx_attend_dev.h"

namespace kvx {
namespace {

template <int kCache>
constexpr bool is8() { return kCache == KVX_FP8_E4M3FN || kCache == KVX_FP8_E5M2; }

template <int kCache>
__device__ __forceinline__ float element(const char* row, int i)
{
    if constexpr (is8<kCache>())
        return value8<kCache == KVX_FP8_E5M2, 0>(reinterpret_cast<const uint8_t*>(row)[i]);
    else
        return value16<kCache == KVX_BF16>(reinterpret_cast<const uint16_t*>(row)[i]);
}

// Whether token i of request r sees slot j, and the distance between them.
__device__ __forceinline__ bool visible(const AttendArgs& a, const Request& rq, int r, int i, int j,
                                        int& distance)
{
    const int tok = rq.first + i;
    const int qp = a.b.positions ? a.b.positions[tok] : rq.ctx + i;
    const int kp = j >= rq.ctx && a.b.positions ? a.b.positions[rq.first + j - rq.ctx] : j;
    distance = qp - kp;
    if (j >= rq.total) return false;
    if (a.prefix && j < a.prefix[r]) return true;
    bool see = true;
    if (j >= rq.ctx) {
        const int k = j - rq.ctx;
        see = a.b.tree ? (a.b.tree[int64_t(tok) * a.b.tree_stride + (k >> 6)] >> (k & 63)) & 1
                       : k <= i;
    }
    return see && (a.window <= 0 || distance < a.window);
}

__device__ __forceinline__ float score(const AttendArgs& a, float dot, int head, int distance)
{
    float x = dot * a.scale;
    if (a.softcap > 0.0f) x = a.softcap * tanhf(x / a.softcap);
    if (a.slopes) x -= a.slopes[head] * static_cast<float>(abs(distance));
    return x;
}

// One wave per (request, KV head, 64 slots): a lane to each slot.
template <bool kBf16, int kCache>
__global__ void __launch_bounds__(64) kvx_weigh_kernel(const AttendArgs a, int tiles)
{
    const int lane = threadIdx.x, D = a.c.dim;
    const int g = (int(blockIdx.x) / tiles) % a.c.hd, r = int(blockIdx.x) / tiles / a.c.hd;
    const Request rq = request_of(a.c, a.b, r);
    const int j = int(blockIdx.x) % tiles * 64 + lane;
    if (j >= rq.total) return;
    const int64_t row = slot_row(a.c, r, j);
    float w = 0.0f;
    if (row >= 0) {
        const char* k = a.c.base + (row + g) * a.c.row_bytes;
        for (int i = 0; i < rq.n; ++i) {
            int dist;
            if (!visible(a, rq, r, i, j, dist)) continue;
            for (int h = g * a.group; h < (g + 1) * a.group; ++h) {
                const uint16_t* q = a.q + int64_t(rq.first + i) * a.q_stride + int64_t(h) * D;
                float dot = 0.0f;
                for (int d = 0; d < D; ++d)
                    dot = __builtin_fmaf(value16<kBf16>(q[d]), element<kCache>(k, d), dot);
                if constexpr (is8<kCache>()) dot *= a.c.scales[row + g];
                const float lse = a.lse[int64_t(rq.first + i) * a.q_heads + h];
                if (lse > -INFINITY) w += __expf(score(a, dot, h, dist) - lse);
            }
        }
    }
    float* out = a.weights + (int64_t(r) * a.c.hd + g) * a.w_stride + j;
    *out = j < rq.ctx ? *out + w : w;
}

// ---- splits joined -------------------------------------------------------------
//
// One workgroup per (token, query head): the sums of its splits, each relative
// to its own reference, brought to the largest and added; always in the same
// order.
template <bool kBf16>
__global__ void __launch_bounds__(256) kvx_join_kernel(const AttendArgs a)
{
    __shared__ float s_part[4][256], s_red[4], s_sum[4];
    const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) >> 6;
    const int64_t at = blockIdx.x, pairs = int64_t(a.b.total_tokens) * a.q_heads;
    const int token = int(at / a.q_heads), head = int(at - int64_t(token) * a.q_heads);
    const int r = request_at(a.b.starts, a.c.num_requests, token);
    if (r < 0 || r >= a.c.num_requests) return;
    const Request rq = request_of(a.c, a.b, r);
    if (token - rq.first >= rq.n) return;
    const float2* const ml = reinterpret_cast<const float2*>(a.part_ml);
    float top = -INFINITY;
    for (int s = threadIdx.x; s < a.splits; s += 256) top = fmaxf(top, ml[s * pairs + at].x);
    for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    if (lane == 0) s_red[wave] = top;
    __syncthreads();
    top = fmaxf(fmaxf(s_red[0], s_red[1]), fmaxf(s_red[2], s_red[3]));
    float acc[4] = {}, total = 0.0f;
    const int D = a.c.dim, d = 4 * lane;
    for (int s = wave; s < a.splits; s += 4) {
        const float2 v = ml[s * pairs + at];
        if (v.x == -INFINITY) continue;
        const float f = __builtin_amdgcn_exp2f(v.x - top);
        total += v.y * f;
        if (d < D) {
            const float4 x = *reinterpret_cast<const float4*>(a.part_o + (s * pairs + at) * D + d);
            acc[0] += x.x * f, acc[1] += x.y * f, acc[2] += x.z * f, acc[3] += x.w * f;
        }
    }
    if (lane == 0) s_sum[wave] = total;
    for (int k = 0; k < 4; ++k) s_part[wave][4 * lane + k] = acc[k];
    __syncthreads();
    if (wave != 0) return;
    total = s_sum[0] + s_sum[1] + s_sum[2] + s_sum[3];
    const float inv = total == 0.0f ? 0.0f : 1.0f / total;
    if (d < D) {
        float x[4];
        for (int k = 0; k < 4; ++k)
            x[k] = (s_part[0][d + k] + s_part[1][d + k] + s_part[2][d + k] + s_part[3][d + k]) * inv;
        *reinterpret_cast<uint2*>(a.out + token * a.out_stride + int64_t(head) * D + d) =
            total == 0.0f ? make_uint2(0, 0) : make_uint2(pack2<kBf16>(x[0], x[1]), pack2<kBf16>(x[2], x[3]));
    }
    if (a.lse && lane == 0)
        a.lse[at] = total == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(total) - kShift<kBf16>) * kLn2;
}

// (split, token, query head) triples, in a multiple of 4
int64_t plan_pairs(const AttendArgs& a, const AttendPlan& p)
{
    return (int64_t(a.b.total_tokens) * a.q_heads * p.splits + 3) & ~int64_t(3);
}

int join(const AttendArgs& a, bool bf, void* stream)
{
    const dim3 grid(uint32_t(a.b.total_tokens) * uint32_t(a.q_heads));
    if (bf)
        kvx_join_kernel<true><<<grid, dim3(256), 0, static_cast<hipStream_t>(stream)>>>(a);
    else
        kvx_join_kernel<false><<<grid, dim3(256), 0, static_cast<hipStream_t>(stream)>>>(a);
    return int(hipGetLastError());
}

template <bool kBf16, int kCache>
int weigh_as(const AttendArgs& a, void* stream)
{
    const int tiles = (a.b.max_context + 63) / 64;
    kvx_weigh_kernel<kBf16, kCache><<<dim3(uint32_t(tiles) * a.c.hd * a.c.num_requests), dim3(64), 0,
                                      static_cast<hipStream_t>(stream)>>>(a, tiles);
    return int(hipGetLastError());
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
                          : launch_rows(a, p, dtype, cache_dtype, stream);
    return err || p.splits == 1 ? err : join(a, bf, stream);
}

int launch_weigh(const AttendArgs& a, int dtype, int cache_dtype, void* stream)
{
    const bool bf = dtype == KVX_BF16;
    switch (cache_dtype) {
    case KVX_FP16: return weigh_as<false, KVX_FP16>(a, stream);
    case KVX_BF16: return weigh_as<true, KVX_BF16>(a, stream);
    case KVX_FP8_E4M3FN: return bf ? weigh_as<true, KVX_FP8_E4M3FN>(a, stream) : weigh_as<false, KVX_FP8_E4M3FN>(a, stream);
    default: return bf ? weigh_as<true, KVX_FP8_E5M2>(a, stream) : weigh_as<false, KVX_FP8_E5M2>(a, stream);
    }
}

AttendPlan attend_plan(const kvx_cache& c, const kvx_batch& b, int32_t q_heads)
{
    AttendPlan p = {};
    p.rows = int(std::min<int64_t>(int64_t(b.max_tokens) * (q_heads / c.num_kv_heads), INT32_MAX));
    p.few = p.rows <= 32;
    p.tile_rows = p.rows <= 16 ? 16 : p.rows <= 32 ? 32 : p.rows <= 64 ? 64 : 128;
    p.row_tiles = (p.rows + p.tile_rows - 1) / p.tile_rows;
    p.chunk = 512;
    if (!p.few) {
        const int64_t groups = int64_t(c.num_requests) * c.num_kv_heads * p.row_tiles;
        const int64_t want = std::max<int64_t>(1, 1024 / groups);
        p.chunk = std::max(512, int((b.max_context + want - 1) / want + 63) & ~63);
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
