// The slots' accumulated attention weight (kvx_weigh).
//
// A wave takes 64 slots of one request and KV head: their keys stay in
// registers as the matrix instructions take them, and the query rows pass by 16
// at a time,
//   S^T = K Q^T,  w[slot] += exp2(x2 - lse2),
// each lane adding up its own query row's weights; the 16 lanes' sums are added
// once at the end, in a fixed order.  Bound by reading K for few rows, by the
// matrix instructions and the exponentials for many.  No two waves write the same
// slot, so nothing is added atomically.
#include <hip/hip_runtime.h>

#include "kvx_attend_dev.h"

namespace kvx {
namespace {

constexpr int kWaves = 4;
constexpr int kKeys = 64;                        // slots of a wave

template <bool kBf16, int kCodes, int DP>
__global__ void __launch_bounds__(64 * kWaves, (DP >= 256 ? 2 : 3)) kvx_weigh_kernel(const AttendArgs a, int tiles)
{
    constexpr bool k8 = kCodes != kCodes16;
    constexpr int kEl = k8 ? 1 : 2, kPieces = DP * kEl / 64, NC = DP / 32;
    __shared__ int64_t s_off[kWaves][kKeys];
    __shared__ int32_t s_pos[kWaves][kKeys];
    __shared__ float s_ks[kWaves][kKeys];
    const int tid = int(threadIdx.x), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n16 = lane & 15, g = lane >> 4;
    const int D = a.c.dim, G = a.group;
    uint32_t u = blockIdx.x;
    const int h = int(u % uint32_t(a.c.hd));
    u /= uint32_t(a.c.hd);
    const int tile = int(u % uint32_t(tiles)), r = int(u / uint32_t(tiles));
    const Request rq = request_of(a.c, a.b, r);
    const int j0 = (tile * kWaves + wave) * kKeys, rows = rq.n * G;
    const bool some = rows > 0 && j0 < rq.total;
    {
        const int j = j0 + lane;
        const int64_t row = some && j < rq.total ? slot_row(a.c, r, j) : -1;
        s_off[wave][lane] = row < 0 ? -1 : (row + h) * a.c.row_bytes;
        s_pos[wave][lane] = a.b.positions && some && j >= rq.ctx && j < rq.total
                                ? a.b.positions[rq.first + j - rq.ctx] : j;
        s_ks[wave][lane] = k8 && row >= 0 ? a.c.scales[row + h] : 0.0f;
    }
    __syncthreads();
    if (!some) return;
    const Range rg = range_of(a, rq, r, 0, rq.n - 1);
    const bool unseen = a.window > 0 && j0 >= rg.pre && j0 + kKeys <= rg.lo;
    if (unseen && j0 + kKeys <= rq.ctx) return;
    const uint64_t valid = __ballot(s_off[wave][lane] >= 0);
    const bool whole = j0 >= rg.all_lo && j0 + kKeys <= rg.all_hi && valid == ~uint64_t(0);

    // keys: slot 16 e + n16, in the element order of 16-byte pieces g, g + 4, ...
    u32x4 k[4][NC];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const char* const row = a.c.base + max(s_off[wave][16 * e + n16], int64_t(0));
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
            const int at = p * 64 + g * 16;
            const u32x4 w = *reinterpret_cast<const u32x4*>(row + (at < a.c.row_bytes ? at : 0));
            if constexpr (k8) {
                k[e][2 * p] = widen8<kBf16, kCodes>(w.x, w.y);
                k[e][2 * p + 1] = widen8<kBf16, kCodes>(w.z, w.w);
            } else {
                k[e][p] = w;
            }
        }
    }
    float ks[4][4], acc[4][4];
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            ks[e][i] = s_ks[wave][16 * e + 4 * g + i];
            acc[e][i] = 0.0f;
        }
    const ScoreArgs sc = score_args(a);

    for (int row0 = 0; row0 < rows; row0 += 16) {
        const int row = row0 + n16;
        const bool live = row < rows;
        const int rr = live ? row : row0;
        const int tok = int(fast_div(uint32_t(rr), a.div_group)), head = h * G + (rr - tok * G);
        const int64_t token = rq.first + tok;
        const uint16_t* const src = a.q + token * a.q_stride + int64_t(head) * D;
        u32x4 q[NC];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int d = k8 ? (c >> 1) * 64 + g * 16 + (c & 1) * 8 : c * 32 + g * 8;
            q[c] = u32x4{0, 0, 0, 0};
            if (d < D) q[c] = *reinterpret_cast<const u32x4*>(src + d);
        }
        const float lse = a.lse[token * a.q_heads + head];
        const float lse2 = lse == -INFINITY ? INFINITY : lse * kLog2e;
        const int qpos = a.b.positions ? a.b.positions[token] : rq.ctx + tok;
        const float slope2 = a.slopes ? a.slopes[head] * kLog2e : 0.0f;
        uint64_t mine = live && lse != -INFINITY ? ~uint64_t(0) : 0;
        if (!whole && mine) mine = seen_of(a, rq, r, tok, qpos, j0, valid);
        mine >>= 4 * g;
        constexpr uint64_t kOwn = 0x000F000F000F000Full;
        const bool all = __all((mine & kOwn) == kOwn);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            f32x4 s = {0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < NC; ++c) s = mfma16<kBf16>(k[e][c], q[c], s);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float dot = k8 ? s[i] * ks[e][i] : s[i];
                const float x = sc.general ? general_score(sc, dot, slope2, qpos - s_pos[wave][16 * e + 4 * g + i])
                                           : dot * sc.c2;
                const float p = __builtin_amdgcn_exp2f(x - lse2);
                acc[e][i] += all || (mine >> (16 * e + i) & 1) ? p : 0.0f;
            }
        }
    }
    // the rows' sums: over the 16 lanes of a group
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float x = acc[e][i];
            x += __shfl_xor(x, 1);
            x += __shfl_xor(x, 2);
            x += __shfl_xor(x, 4);
            x += __shfl_xor(x, 8);
            acc[e][i] = x;
        }
    // lane (n16, g) writes slot 16 (n16 / 4) + 4 g + n16 % 4
    float w = 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n16 == 4 * e + i) w = acc[e][i];
    const int j = j0 + 16 * (n16 >> 2) + 4 * g + (n16 & 3);
    if (j < rq.total) {
        float* const out = a.weights + (int64_t(r) * a.c.hd + h) * a.w_stride + j;
        *out = j < rq.ctx ? *out + w : w;
    }
}

template <bool kBf16, int kCodes, int DP>
int go(const AttendArgs& a, void* stream)
{
    const int tiles = (a.b.max_context + kWaves * kKeys - 1) / (kWaves * kKeys);
    kvx_weigh_kernel<kBf16, kCodes, DP>
        <<<dim3(uint32_t(tiles) * a.c.hd * a.c.num_requests), dim3(64 * kWaves), 0,
           static_cast<hipStream_t>(stream)>>>(a, tiles);
    return int(hipGetLastError());
}

template <bool kBf16, int kCodes>
int pick(const AttendArgs& a, void* stream)
{
    if (a.c.dim <= 64) return go<kBf16, kCodes, 64>(a, stream);
    return a.c.dim <= 128 ? go<kBf16, kCodes, 128>(a, stream) : go<kBf16, kCodes, 256>(a, stream);
}

}  // namespace

int launch_weigh(const AttendArgs& a, int dtype, int cache_dtype, void* stream)
{
    const bool bf = dtype == KVX_BF16;
    switch (cache_dtype) {
    case KVX_FP8_E4M3FN: return bf ? pick<true, kCodesE4m3>(a, stream) : pick<false, kCodesE4m3>(a, stream);
    case KVX_FP8_E5M2: return bf ? pick<true, kCodesE5m2>(a, stream) : pick<false, kCodesE5m2>(a, stream);
    default: return bf ? pick<true, kCodes16>(a, stream) : pick<false, kCodes16>(a, stream);
    }
}

}  // namespace kvx
