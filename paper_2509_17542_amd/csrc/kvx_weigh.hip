// The slots' accumulated attention weight (kvx_weigh).
//
// A wave takes 32 or 64 slots of one request and KV head: their rows go to LDS of
// its own, whole, 32 at a time, and from there to the matrix instructions; the
// query rows pass by 16 at a time,
//   S^T = K Q^T,  w[slot] += exp2(x2 - lse2),
// each lane adding up its own query row's weights; the 16 lanes' sums are added
// at the end, in a fixed order.  For 16 rows or fewer a wave is a chain (places,
// rows, products, weights), bound by how many waves a SIMD holds: 32 keys that
// stay in LDS leave registers for four (32 requests of 512..4096 slots, e5m2: 24
// us; 30 with 64 keys in registers).  For more it is bound by the matrix
// instructions and the exponentials, and 64 keys in registers serve all rows
// (the last 32 tokens of two prompts of 16000..32000 slots, 128 rows: 42 us,
// 2.5 TB/s and 304 TFLOP/s; in short runs 45, and 68 the other way).  No two
// waves write the same slot, so nothing is added atomically.
#include <hip/hip_runtime.h>

#include "kvx_attend_dev.h"

namespace kvx {
namespace {

constexpr int kWaves = 4;

// kHalves: 32 slots each; two are held in registers
template <bool kBf16, int kCodes, int DP, int kScores, int kHalves>
__global__ void __launch_bounds__(64 * kWaves, (DP >= 256 ? 2 : kHalves == 2 ? 3 : 4))
    kvx_weigh_kernel(const AttendArgs a, int tiles)
{
    constexpr int kKeys = 32 * kHalves, kTiles16 = 2 * kHalves;
    constexpr bool kHeld = kHalves == 2, kOther = kScores != kPlain;
    constexpr bool k8 = kCodes != kCodes16;
    constexpr int kEl = k8 ? 1 : 2, NC = DP / 32;
    constexpr int kRow = DP * kEl, kRowPieces = kRow / 16, kLoads = 32 * kRow / 1024;
    __shared__ __attribute__((aligned(16))) char s_k[kWaves][32 * kRow];
    __shared__ int64_t s_off[kWaves][kKeys];
    __shared__ float s_ks[kWaves][kKeys];
    __shared__ int32_t s_pos[kWaves][kOther ? kKeys : 1];
    const int tid = int(threadIdx.x), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n16 = lane & 15, g = lane >> 4;
    const int D = a.c.dim, G = a.group;
    uint32_t u = blockIdx.x;
    const int h = int(u % uint32_t(a.c.hd));
    u /= uint32_t(a.c.hd);
    const int tile = int(u % uint32_t(tiles)), r = int(u / uint32_t(tiles));
    const Request rq = request_of(a.c, a.b, r);
    const int j0 = (tile * kWaves + wave) * kKeys, rows = rq.n * G;
    if (rows == 0 || j0 >= rq.total) return;     // waves share nothing
    const int64_t my_row = lane < kKeys && j0 + lane < rq.total ? slot_row(a.c, r, j0 + lane) : -1;
    const uint64_t valid = __ballot(my_row >= 0);
    if (lane < kKeys) {
        // a slot that lies in no page reads the plane's first row, and is masked
        s_off[wave][lane] = my_row < 0 ? 0 : (my_row + h) * a.c.row_bytes;
        if constexpr (k8) s_ks[wave][lane] = my_row < 0 ? 0.0f : a.c.scales[my_row + h];
        if constexpr (kOther) s_pos[wave][lane] = place_of(a, rq, j0 + lane);
    }
    // a wave's LDS is its own and its accesses stay in order: nothing to wait for
    __builtin_amdgcn_wave_barrier();
    const Range rg = range_of(a, rq, r, 0, rq.n - 1);
    // what no token sees keeps its weight, new tokens' slots apart
    if (a.window > 0 && j0 >= rg.pre && j0 + kKeys <= rg.lo && j0 + kKeys <= rq.ctx) return;
    constexpr uint64_t kAll = ~uint64_t(0) >> (64 - kKeys);
    const bool whole = j0 >= rg.all_lo && j0 + kKeys <= rg.all_hi && valid == kAll;

    // Rows are read whole, 1 KB an instruction; piece p of slot s lies at place
    // p ^ turn_of(s), so that 16 slots' pieces of one number lie in different banks.
    auto turn_of = [](int s) { return kRow >= 256 ? s & 15 : (s / (256 / kRow)) & (kRowPieces - 1); };
    u32x4 raw[kHalves][kLoads];
#pragma unroll
    for (int half = 0; half < kHalves; ++half)
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int s = (i * 64 + lane) / kRowPieces, piece = (i * 64 + lane) % kRowPieces * 16;
            raw[half][i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(
                a.c.base + s_off[wave][32 * half + s] + (piece < a.c.row_bytes ? piece : 0)));
        }

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
    Rows now;
    read_rows(0, now);
    // of each 16 lanes the first 4 kTiles16 write a slot: 16 (i / 4) + 4 g + i % 4, i being the lane's
    // bits turned round
    constexpr int kWriters = 4 * kTiles16, kBits = kHeld ? 4 : 3;
    const int i16 = int(__builtin_bitreverse32(uint32_t(n16 & (kWriters - 1))) >> (32 - kBits));
    const int j = j0 + 16 * (i16 >> 2) + 4 * g + (i16 & 3);
    float* const out = a.weights + (int64_t(r) * a.c.hd + h) * a.w_stride + min(j, rq.total - 1);
    const float old = *out;
    const ScoreArgs sc = score_args(a);
    // the c-th operand of 16 slots of the half that lies in LDS
    auto operand = [&](int e, int c) {
        const int slot = 16 * e + n16;
        const u32x4 w = *reinterpret_cast<const u32x4*>(
            s_k[wave] + slot * kRow + ((4 * (k8 ? c >> 1 : c) + g) ^ turn_of(slot)) * 16);
        if constexpr (k8) return c & 1 ? widen8<kBf16, kCodes>(w.z, w.w) : widen8<kBf16, kCodes>(w.x, w.y);
        return w;
    };
    u32x4 held[kHeld ? kTiles16 : 1][NC];
#pragma unroll
    for (int half = 0; half < kHalves; ++half) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int s = (i * 64 + lane) / kRowPieces, place = ((i * 64 + lane) % kRowPieces) ^ turn_of(s);
            *reinterpret_cast<u32x4*>(s_k[wave] + s * kRow + place * 16) = raw[half][i];
        }
        if constexpr (kHeld) {
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int c = 0; c < NC; ++c) held[2 * half + e][c] = operand(e, c);
        }
    }
    float ks[kTiles16][4], v[4 * kTiles16] = {};
#pragma unroll
    for (int e = 0; e < kTiles16; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i) ks[e][i] = k8 ? s_ks[wave][16 * e + 4 * g + i] * sc.c2 : sc.c2;

    for (int row0 = 0; row0 < rows; row0 += 16) {
        Rows next;
        if (rows > 16) read_rows(row0 + 16 < rows ? row0 + 16 : 0, next);
        const float lse2 = now.lse == -INFINITY ? INFINITY : now.lse * kLog2e;
        const float slope2 = kOther && a.slopes ? a.slopes[now.head] * kLog2e : 0.0f;
        uint64_t mine = now.live && now.lse != -INFINITY ? ~uint64_t(0) : 0;
        if (!whole && mine) mine = seen_of(a, rq, r, now.tok, now.qpos, j0, valid);
        mine >>= 4 * g;
        constexpr uint64_t kOwn = 0x000F000F000F000Full & kAll;
        const bool all = __all((mine & kOwn) == kOwn);
#pragma unroll
        for (int e = 0; e < kTiles16; ++e) {
            f32x4 s = {0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < NC; ++c) s = mfma16<kBf16>(kHeld ? held[kHeld ? e : 0][c] : operand(e, c), now.q[c], s);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float x = s[i] * ks[e][i];
                if constexpr (kOther)
                    x = general_score<kScores>(sc, k8 ? s[i] * s_ks[wave][16 * e + 4 * g + i] : s[i], slope2,
                                               now.qpos - s_pos[wave][16 * e + 4 * g + i]);
                const float p = __builtin_amdgcn_exp2f(x - lse2);
                v[4 * e + i] += all || (mine >> (16 * e + i) & 1) ? p : 0.0f;
            }
        }
        if (rows > 16) now = next;
    }
    // The rows' sums, over the 16 lanes of a group: in each step a lane gives half of its values
    // away and adds its partner's to the other half, so that one is left, that of its slot.
#pragma unroll
    for (int s = 0; s < kBits; ++s) {
        const bool upper = n16 >> s & 1;
        const int half = (kWriters / 2) >> s;
#pragma unroll
        for (int i = 0; i < half; ++i) {
            const float kept = upper ? v[i + half] : v[i], given = upper ? v[i] : v[i + half];
            v[i] = kept + __shfl_xor(given, 1 << s);
        }
    }
    const float w = kHeld ? v[0] : v[0] + __shfl_xor(v[0], 8);
    if (n16 < kWriters && j < rq.total) *out = j < rq.ctx ? old + w : w;
}

// more than 16 query rows: 64 slots a wave, else 32
int halves_of(int32_t max_tokens, int32_t group) { return int64_t(max_tokens) * group > 16 ? 2 : 1; }

int tiles_of(int32_t max_context, int halves) { return (max_context + kWaves * 32 * halves - 1) / (kWaves * 32 * halves); }

template <bool kBf16, int kCodes, int DP, int kScores, int kHalves>
int go_as(const AttendArgs& a, void* stream)
{
    const int tiles = tiles_of(a.b.max_context, kHalves);
    return launch_kernel(kvx_weigh_kernel<kBf16, kCodes, DP, kScores, kHalves>,
                         int64_t(tiles) * a.c.hd * a.c.num_requests, 64 * kWaves, stream, a, tiles);
}

template <bool kBf16, int kCodes, int DP, int kScores>
int go_by(const AttendArgs& a, void* stream)
{
    return halves_of(a.b.max_tokens, a.group) == 2 ? go_as<kBf16, kCodes, DP, kScores, 2>(a, stream)
                                                   : go_as<kBf16, kCodes, DP, kScores, 1>(a, stream);
}

template <bool kBf16, int kCodes, int DP>
int go(const AttendArgs& a, void* stream)
{
    switch (scores_of(a)) {
    case kWide: return go_by<kBf16, kCodes, DP, kWide>(a, stream);
    case kGeneral: return go_by<kBf16, kCodes, DP, kGeneral>(a, stream);
    default: return go_by<kBf16, kCodes, DP, kPlain>(a, stream);
    }
}

template <bool kBf16, int kCodes>
int pick(const AttendArgs& a, void* stream)
{
    if (a.c.dim <= 64) return go<kBf16, kCodes, 64>(a, stream);
    return a.c.dim <= 128 ? go<kBf16, kCodes, 128>(a, stream) : go<kBf16, kCodes, 256>(a, stream);
}

}  // namespace

double weigh_threads(const kvx_cache& c, const kvx_batch& b, int32_t q_heads)
{
    const int tiles = tiles_of(b.max_context, halves_of(b.max_tokens, q_heads / c.num_kv_heads));
    return double(tiles) * c.num_kv_heads * c.num_requests * (64 * kWaves);
}

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
