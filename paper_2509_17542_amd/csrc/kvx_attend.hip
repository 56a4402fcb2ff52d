// kvx_attend: how a call is cut into workgroups, and the join of its splits.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "kvx_attend_dev.h"

namespace kvx {
namespace {

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
