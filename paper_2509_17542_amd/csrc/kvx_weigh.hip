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
    constexpr int kRow = DP * kEl, kRowPieces = kRow / 16, kLoads = 32 * kRow / 1024;
    __shared__ __attribute__((aligned(16))) char s_k[kWaves][32 * kRow];
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

    // Query rows: a lane takes row n16 of 16; the next 16 are on their way while these pass.
    struct Rows {
        u32x4 q[NC];
        float lse;
        int tok, head, qpos;
        bool live;
    };
    auto read_rows = [&](int row0, Rows& x) {
        const int row = row0 + n16;
        x.live = row < rows;
        const int rr = x.live ? row : 0;
        x.tok = int(fast_div(uint32_t(rr), a.div_group));
        x.head = h * G + (rr - x.tok * G);
        const int64_t token = rq.first + x.tok;
        const uint16_t* const src = a.q + token * a.q_stride + int64_t(x.head) * D;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int d = k8 ? (c >> 1) * 64 + g * 16 + (c & 1) * 8 : c * 32 + g * 8;
            x.q[c] = *reinterpret_cast<const u32x4*>(src + (d < D ? d : 0));
            if (d >= D) x.q[c] = u32x4{0, 0, 0, 0};
        }
        x.lse = a.lse[token * a.q_heads + x.head];
        x.qpos = a.b.positions ? a.b.positions[token] : rq.ctx + x.tok;
    };
    // lane (n16, g) writes slot 16 (n16 / 4) + 4 g + n16 % 4
    const int j = j0 + 16 * (n16 >> 2) + 4 * g + (n16 & 3);
    float* const out = a.weights + (int64_t(r) * a.c.hd + h) * a.w_stride + min(j, rq.total - 1);
    const float old = *out;
    Rows now;
    read_rows(0, now);

    // Keys: slot 16 e + n16, in the element order of 16-byte pieces g, g + 4, ...  Rows are
    // read whole, 1 KB an instruction, and turned round in LDS of the wave's own, 32 slots
    // at a time; piece p of slot s lies at place p ^ turn_of(s), so that 16 slots' pieces
    // of one number lie in different banks.
    auto turn_of = [](int s) { return kRow >= 256 ? s & 15 : (s / (256 / kRow)) & (kRowPieces - 1); };
    u32x4 raw[2][kLoads];
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int s = (i * 64 + lane) / kRowPieces, piece = (i * 64 + lane) % kRowPieces * 16;
            raw[half][i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(
                a.c.base + max(s_off[wave][32 * half + s], int64_t(0)) + (piece < a.c.row_bytes ? piece : 0)));
        }
    u32x4 k[4][NC];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int s = (i * 64 + lane) / kRowPieces, place = ((i * 64 + lane) % kRowPieces) ^ turn_of(s);
            *reinterpret_cast<u32x4*>(s_k[wave] + s * kRow + place * 16) = raw[half][i];
        }
#pragma unroll
        for (int e = 2 * half; e < 2 * half + 2; ++e)
#pragma unroll
            for (int p = 0; p < kPieces; ++p) {
                const int s = 16 * (e & 1) + n16;
                const u32x4 w = *reinterpret_cast<const u32x4*>(s_k[wave] + s * kRow + ((4 * p + g) ^ turn_of(s)) * 16);
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
        Rows next;
        read_rows(row0 + 16 < rows ? row0 + 16 : row0, next);
        const float lse2 = now.lse == -INFINITY ? INFINITY : now.lse * kLog2e;
        const float slope2 = a.slopes ? a.slopes[now.head] * kLog2e : 0.0f;
        uint64_t mine = now.live && now.lse != -INFINITY ? ~uint64_t(0) : 0;
        if (!whole && mine) mine = seen_of(a, rq, r, now.tok, now.qpos, j0, valid);
        mine >>= 4 * g;
        constexpr uint64_t kOwn = 0x000F000F000F000Full;
        const bool all = __all((mine & kOwn) == kOwn);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            f32x4 s = {0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < NC; ++c) s = mfma16<kBf16>(k[e][c], now.q[c], s);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float dot = k8 ? s[i] * ks[e][i] : s[i];
                const float x = sc.general ? general_score(sc, dot, slope2, now.qpos - s_pos[wave][16 * e + 4 * g + i])
                                           : dot * sc.c2;
                const float p = __builtin_amdgcn_exp2f(x - lse2);
                acc[e][i] += all || (mine >> (16 * e + i) & 1) ? p : 0.0f;
            }
        }
        now = next;
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
    float w = 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n16 == 4 * e + i) w = acc[e][i];
    if (j < rq.total) *out = j < rq.ctx ? old + w : w;
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
