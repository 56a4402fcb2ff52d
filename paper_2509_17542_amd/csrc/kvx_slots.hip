// gfx950 kernels that write and move rows of the paged cache: kvx_append (the
// new tokens' rows, with rotary positions), kvx_evict (selection by weight, then
// the move of what stays, a head's rows at a time) and kvx_commit (the move of a
// path's rows, all heads at a time).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "kvx_ops_dev.h"

namespace kvx {
namespace {

constexpr int kWg = 256;

// ---- append ------------------------------------------------------------------

// Maximum over each aligned group of 2^lg lanes, lg <= 5, all of them active.
__device__ __forceinline__ float lanes_max(float m, int lg)
{
    for (int o = 1; o < (1 << lg); o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
    return m;
}

// x / s -> 8-bit code: a NaN keeps its sign, a zero scale gives signed zeros,
// finite values saturate (only rounding of the quotient can pass the largest).
template <bool kE5>
__device__ __forceinline__ uint32_t code8(float x, float s)
{
    const uint32_t sign = (__float_as_uint(x) >> 24) & 0x80u;
    if (x != x) return sign | 0x7Fu;
    if (s == 0.0f) return sign;
    const float q = __builtin_fabsf(x) / s;
    if (q != q) return sign | 0x7Fu;
    const float c = fminf(q, kE5 ? 57344.0f : 448.0f);
    uint32_t code;
    if constexpr (kE5)
        code = uint32_t(__builtin_amdgcn_cvt_pk_bf8_f32(c, c, 0, false)) & 0x7Fu;
    else
        code = uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(c, c, 0, false)) & 0x7Fu;
    return sign | code;
}

enum Pairing : int { kHalves = 0, kInterleaved = 1, kAnyHalves = 2 };

// 8 elements of 16 bits -> fp32
template <bool kBf16>
__device__ __forceinline__ void widen(const uint4& w, float (&x)[8])
{
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = value16<kBf16>((u[e >> 1] >> (16 * (e & 1))) & 0xFFFFu);
}

template <bool kBf16>
__device__ __forceinline__ uint4 narrow(const float (&x)[8])
{
    uint32_t u[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) u[k] = bits16<kBf16>(x[2 * k]) | bits16<kBf16>(x[2 * k + 1]) << 16;
    return make_uint4(u[0], u[1], u[2], u[3]);
}

// A workgroup takes a token: its turns (cosine and sine of the fp32 angles,
// reduced in fp64 to a fraction of a turn) go to LDS once for all heads, and its
// place in the cache is looked up meanwhile.  A power-of-two group of lanes then
// covers a head, 8 elements (16 bytes) a lane, whose turns stay in registers for
// all of the token's heads; the element that a turn pairs with lies in the lane
// (interleaved) or is read again, out of the cache (halves; pairs that do not fill
// whole lanes element by element).  Bound by memory for prompts and by its chain
// of lookups for single tokens.  Prompts of 500..3000 tokens, three axes, into an
// fp8 cache (250 MB) take 61 us, 4.1 TB/s, on buffers that change from call to call;
// on the same ones 53, and 60 into a bf16 cache, with four tokens a workgroup 59 and 70.
template <bool kBf16, int kCache, int kPairing>
__global__ void __launch_bounds__(kWg) kvx_append_kernel(const AppendArgs a)
{
    __shared__ float2 s_turn[128];
    __shared__ int64_t s_row;
    const int t = int(blockIdx.x), wave = int(threadIdx.x) >> 6;
    const int D = a.c.dim, P = a.pairs, N = a.b.total_tokens;
    for (int i = threadIdx.x; i < P; i += kWg) {
        int axis = 0;
#pragma unroll
        for (int s = 0; s < 3; ++s) axis += i >= a.sec_end[s];
        const float pos = static_cast<float>(a.positions[int64_t(axis) * N + t]);
        const double turns = double(pos * a.inv_freq[i]) * 0.15915494309189533577;
        float sn, cs;
        sincospif(2.0f * static_cast<float>(turns - rint(turns)), &sn, &cs);
        s_turn[i] = make_float2(cs, sn);
    }
    if (wave == kWg / 64 - 1) {                  // the pairs are the first waves'
        int64_t row = -1;
        const int r = request_at(a.b.starts, a.c.num_requests, t);
        if (r >= 0 && r < a.c.num_requests) {
            const Request rq = request_of(a.c, a.b, r);
            const int j = rq.ctx + (t - rq.first);
            if (t - rq.first < rq.n && j < rq.total) row = slot_row(a.c, r, j);
        }
        if ((threadIdx.x & 63) == 0) s_row = row;
    }
    __syncthreads();
    const int per = 1 << a.lg_row, lane = int(threadIdx.x) & (per - 1), e0 = lane * 8;
    const int rows = a.q_heads + 2 * a.c.hd;
    const bool in_row = e0 < D;
    const int64_t row = s_row;
    // the turns of this lane's elements: x cs + y sn, the sign of sn with it
    float cs[8], sn[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int i = e0 + e;
        cs[e] = 1.0f, sn[e] = 0.0f;
        if (i < 2 * P) {
            const bool second = kPairing == kInterleaved ? i & 1 : i >= P;
            const float2 x = s_turn[kPairing == kInterleaved ? i >> 1 : second ? i - P : i];
            cs[e] = x.x;
            sn[e] = second ? x.y : -x.y;
        }
    }
    const bool turned = e0 < 2 * P;              // and so in the row
    const int other = kPairing == kHalves && turned ? (e0 >= P ? e0 - P : e0 + P) : e0;
    for (int h = int(threadIdx.x) >> a.lg_row; h < rows; h += kWg >> a.lg_row) {
        const bool is_q = h < a.q_heads, is_v = h >= a.q_heads + a.c.hd;
        const uint16_t* const src = is_q ? a.q + t * a.q_stride + int64_t(h) * D
                                  : is_v ? a.v + t * a.v_stride + int64_t(h - a.q_heads - a.c.hd) * D
                                         : a.k + t * a.k_stride + int64_t(h - a.q_heads) * D;
        // lanes past the row's end hold zeros: the row's maximum takes all of its group
        float x[8] = {};
        if (in_row) widen<kBf16>(*reinterpret_cast<const uint4*>(src + e0), x);
        if (!is_v && turned) {
            float y[8];
            if constexpr (kPairing == kInterleaved) {
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = x[e ^ 1];
            } else if constexpr (kPairing == kHalves) {
                widen<kBf16>(*reinterpret_cast<const uint4*>(src + other), y);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int i = e0 + e;
                    y[e] = i < 2 * P ? value16<kBf16>(src[i >= P ? i - P : i + P]) : 0.0f;
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e0 + e < 2 * P) x[e] = x[e] * cs[e] + y[e] * sn[e];
        }
        if (is_q) {
            // q_out may be q: the head's lanes, all of one wave, have read it
            __builtin_amdgcn_wave_barrier();
            if (in_row)
                *reinterpret_cast<uint4*>(a.q_out + t * a.q_out_stride + int64_t(h) * D + e0) = narrow<kBf16>(x);
            continue;
        }
        const int kv = is_v ? 1 : 0, head = h - a.q_heads - (is_v ? a.c.hd : 0);
        char* const dst = a.c.base + kv * a.c.plane_bytes + (row + head) * a.c.row_bytes;
        if constexpr (kCache == KVX_FP16 || kCache == KVX_BF16) {
            if (row >= 0 && in_row) *reinterpret_cast<uint4*>(dst + e0 * 2) = narrow<kCache == KVX_BF16>(x);
        } else {
            constexpr bool kE5 = kCache == KVX_FP8_E5M2;
            float m = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) m = fmaxf(m, __builtin_fabsf(x[e]));  // a NaN takes no part
            m = lanes_max(m, a.lg_row);
            const float s = m / (kE5 ? 57344.0f : 448.0f);
            uint32_t w[2] = {0, 0};
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e >> 2] |= code8<kE5>(x[e], s) << (8 * (e & 3));
            if (row >= 0 && in_row) {
                *reinterpret_cast<uint2*>(dst + e0) = make_uint2(w[0], w[1]);
                if (lane == 0) a.c.scales[kv * a.c.plane_scales + row + head] = s;
            }
        }
    }
}

// ---- evict: selection ---------------------------------------------------------

// A weight's place in the order that eviction goes by: larger weights have
// larger keys, -0 and 0 the same, every NaN the largest.
__device__ __forceinline__ uint32_t weight_key(float w)
{
    if (w != w) return 0xFFFFFFFFu;
    const uint32_t u = __float_as_uint(w == 0.0f ? 0.0f : w);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// One workgroup per (layer, request, head).  The weight of the last slot that
// stays is found by its key, 11, 11 and 10 bits at a time: a histogram of the
// candidates that agree with the bits found so far, walked from the top.  Then
// one pass in slot order writes what stays; of the slots that tie with that
// weight the first ones, which takes a second count only where not all of them
// stay.  The weights are read four times, all but the first from the L2.
template <int kThreads_>
__global__ void __launch_bounds__(kThreads_) kvx_select_kernel(const EvictArgs a)
{
    constexpr int kW = kThreads_ / 64, kBins = 2048, kPer = kBins / kThreads_;
    constexpr int kEach = 4;                     // slots of a thread at once
    __shared__ uint32_t s_hist[kBins];
    __shared__ uint32_t s_part[2][kW];
    __shared__ uint32_t s_bin, s_left, s_same;
    const int tid = int(threadIdx.x), lane = tid & 63, wave = tid >> 6;
    const int lrh = int(blockIdx.x);
    const int r = (lrh / a.c.hd) % a.c.num_requests;
    const int T = min(min(max(a.lens[r], 0), a.max_len), a.c.row_slots);
    const int keep = min(T, a.budget);
    const float* w = a.weights + int64_t(lrh) * a.w_stride;
    float* w_out = a.weights_out + int64_t(lrh) * a.w_stride;
    int32_t* kept = a.kept + int64_t(lrh) * a.budget;
    if (lrh < a.c.num_requests * a.c.hd && lrh % a.c.hd == 0 && tid == 0) a.new_lens[r] = keep;
    if (T <= a.budget) {
        for (int i = tid; i < a.budget; i += kThreads_) {
            if (i < T && w_out != w) w_out[i] = w[i];
            kept[i] = i < T ? i : -1;
        }
        return;
    }
    const int lo = a.sink, hi = T - a.recent;    // candidates; sink + recent <= budget < T
    uint32_t left = uint32_t(a.budget - a.sink - a.recent), same = 0;
    uint32_t key = 0;                            // bits found so far
    const bool any = left != 0;
    if (any) {
        for (int step = 0; step < 3; ++step) {
            const int shift = step == 0 ? 21 : step == 1 ? 10 : 0;
            const uint32_t mask = step == 2 ? 1023u : 2047u;
            for (int b = tid; b < kBins; b += kThreads_) s_hist[b] = 0;
            __syncthreads();
            const int above = step == 0 ? 32 : step == 1 ? 21 : 10;
            for (int j0 = lo + tid; j0 < hi; j0 += kEach * kThreads_) {
                float x[kEach];
#pragma unroll
                for (int e = 0; e < kEach; ++e) x[e] = w[min(j0 + e * kThreads_, hi - 1)];
#pragma unroll
                for (int e = 0; e < kEach; ++e) {
                    const uint32_t k = weight_key(x[e]);
                    if (j0 + e * kThreads_ < hi && (step == 0 || (k >> above) == (key >> above)))
                        atomicAdd(&s_hist[(k >> shift) & mask], 1u);
                }
            }
            __syncthreads();
            // thread i holds kPer bins from the top down
            uint32_t mine[kPer], sum = 0;
#pragma unroll
            for (int b = 0; b < kPer; ++b) sum += mine[b] = s_hist[kBins - 1 - (tid * kPer + b)];
            uint32_t upto = sum;
            for (int o = 1; o < 64; o <<= 1) {
                const uint32_t u = __shfl_up(upto, o);
                if (lane >= o) upto += u;
            }
            if (lane == 63) s_part[0][wave] = upto;
            __syncthreads();
            for (int k = 0; k < wave; ++k) upto += s_part[0][k];
            uint32_t before = upto - sum;
#pragma unroll
            for (int b = 0; b < kPer; ++b) {
                if (before < left && before + mine[b] >= left) {
                    s_bin = kBins - 1 - (tid * kPer + b);
                    s_left = left - before;
                    s_same = mine[b];
                }
                before += mine[b];
            }
            __syncthreads();
            key |= s_bin << shift;
            left = s_left;
            same = s_same;
            __syncthreads();
        }
    }
    // all slots above `key` stay and the first `left` of the `same` that equal it
    const bool all_ties = same == left;
    uint32_t ties = 0, out = 0;
    int turn = 0;
    // Counts flags over the workgroup in slot order, kEach consecutive slots a thread: how many
    // lie before this thread's, and in all.
    auto count = [&](const bool (&flag)[kEach], uint32_t& total) {
        const uint64_t below = (uint64_t(1) << lane) - 1;
        uint32_t before = 0, all = 0;
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const uint64_t m = __ballot(flag[e]);
            before += uint32_t(__popcll(m & below));
            all += uint32_t(__popcll(m));
        }
        uint32_t* const part = s_part[turn];
        turn ^= 1;                               // the other half may still be read
        if (lane == 0) part[wave] = all;
        __syncthreads();
        total = 0;
#pragma unroll
        for (int k = 0; k < kW; ++k) {
            before += k < wave ? part[k] : 0u;
            total += part[k];
        }
        return before;
    };
    constexpr int kRound = kEach * kThreads_;
    float x[kEach], next[kEach];
#pragma unroll
    for (int e = 0; e < kEach; ++e) x[e] = w[min(kEach * tid + e, T - 1)];
    for (int j0 = 0; j0 < T; j0 += kRound) {
        const int j = j0 + kEach * tid;
        // read ahead of this round's writes: w_out may be w, and they lie below
#pragma unroll
        for (int e = 0; e < kEach; ++e) next[e] = w[min(j + kRound + e, T - 1)];
        bool stay[kEach], tie[kEach];
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const bool cand = j + e >= lo && j + e < hi;
            const uint32_t k = weight_key(x[e]);
            tie[e] = any && cand && k == key;
            stay[e] = j + e < T && (!cand || (any && k > key) || (all_ties && tie[e]));
        }
        if (!all_ties) {
            uint32_t n;
            uint32_t rank = count(tie, n) + ties;
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
                stay[e] |= tie[e] && rank < left;
                rank += tie[e];
            }
            ties += n;
        }
        uint32_t n;
        uint32_t at = count(stay, n) + out;
        out += n;
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            if (stay[e]) {
                kept[at] = j + e;
                w_out[at] = x[e];                // at <= j + e: read by every thread already
                ++at;
            }
            x[e] = next[e];
        }
    }
}

// ---- rows move up -------------------------------------------------------------
//
// A row never moves down (its source is at or above its target, both ascend), so
// rows may move in place in order, a group at a time: all of a group's rows are
// read before any of it is written, and a write can only hit rows that this or
// an earlier group has read.  Pieces of 16 bytes, a power-of-two number of lanes
// to a row, kHold pieces a lane in flight.  Bound by memory.
constexpr int kHold = 8;

typedef uint32_t piece_t __attribute__((ext_vector_type(4)));

// What a lane holds of a group.
struct Held {
    piece_t x[kHold];
    float s[kHold];
    int64_t to[kHold];                           // row it goes to, -1: none
};

// Every load of `v` has returned: the compiler waits for those alone, not for
// stores that are younger.
__device__ __forceinline__ void arrived(Held& v)
{
#pragma unroll
    for (int k = 0; k < kHold; ++k) __asm__ volatile("" : "+v"(v.x[k]), "+v"(v.s[k]));
}

// Eviction: one workgroup per (layer, k/v, request, head), whose kept slots are
// its own.  The next group's rows are read before this one's are written, and
// the places of the one after that looked up meanwhile.  Rows of whole 256 bytes
// are read non-temporal (kOnce): a prompt of 16001 slots cut to 2048 in 32 layers
// takes 127 us so and 148 without, both with a slower selection (now 117, the move
// 93 of it, 5.8 TB/s; bf16, rows of 256 bytes); an fp8 batch, rows of 128 bytes, 99
// and 91 (the move 78, 5.3 TB/s).  All of this on the same buffers in every call, what
// the last one wrote still in the memory-side cache; on changing ones 143 and 114.
template <bool kOnce>
__global__ void __launch_bounds__(kWg) kvx_move_kernel(const MoveArgs a)
{
    __shared__ int64_t s_src[2][kWg], s_dst[2][kWg];
    const int tid = int(threadIdx.x), H = a.c.hd, R = a.c.num_requests;
    int u = int(blockIdx.x);
    const int h = u % H;
    u /= H;
    const int r = u % R;
    u /= R;
    const int kv = u & 1, layer = u >> 1;
    const int T = min(min(max(a.lens[r], 0), a.max_len), a.c.row_slots);
    const int rows = T > a.budget ? a.budget : 0;
    if (rows == 0) return;
    const int32_t* const index = a.kept + ((int64_t(layer) * R + r) * H + h) * a.budget;
    const int64_t plane = int64_t(2) * layer + kv;
    char* const base = a.c.base + plane * a.c.plane_bytes;
    float* const scales = a.c.scales ? a.c.scales + plane * a.c.plane_scales : nullptr;
    const int pieces = a.c.row_bytes >> 4, lg = a.lg_lanes;
    const int sets = min(kWg >> lg, kWg / kHold), group = sets * kHold;
    const int set = tid >> lg, piece = tid & ((1 << lg) - 1);
    const bool mine = set < sets && piece < pieces;
    const int64_t at = min(piece, pieces - 1) * 16;

    auto look_up = [&](int i0, int side) {
        if (tid < group) {
            const int i = i0 + tid;
            int64_t src = -1, dst = -1;
            if (i < rows) {
                const int from = index[i];
                if (from > i && from < a.c.row_slots) {
                    src = slot_row(a.c, r, from);
                    dst = slot_row(a.c, r, i);
                }
            }
            s_src[side][tid] = src < 0 || dst < 0 ? 0 : src + h;   // one that stays reads the first row
            s_dst[side][tid] = src < 0 || dst < 0 ? -1 : dst + h;
        }
    };
    auto load = [&](int side, Held& v) {
#pragma unroll
        for (int k = 0; k < kHold; ++k) {
            const int row = min(set, sets - 1) + k * sets;
            const int64_t src = s_src[side][row];
            v.to[k] = mine ? s_dst[side][row] : -1;
            const piece_t* const from = reinterpret_cast<const piece_t*>(base + src * a.c.row_bytes + at);
            v.x[k] = kOnce ? __builtin_nontemporal_load(from) : *from;
            v.s[k] = scales ? scales[src] : 0.0f;
        }
    };
    auto store = [&](const Held& v) {
#pragma unroll
        for (int k = 0; k < kHold; ++k)
            if (v.to[k] >= 0) {
                *reinterpret_cast<piece_t*>(base + v.to[k] * a.c.row_bytes + at) = v.x[k];
                if (scales && piece == 0) scales[v.to[k]] = v.s[k];
            }
    };
    Held now, next;
    look_up(0, 0);
    look_up(group, 1);
    __syncthreads();
    load(0, now);
    int side = 1;
    for (int i0 = 0; i0 < rows; i0 += group, side ^= 1) {
        arrived(now);
        __syncthreads();                         // all of this group is in registers
        load(side, next);
        // the places of the group after that go where this one's were
        look_up(i0 + 2 * group, side ^ 1);
        store(now);
        now = next;
    }
}

// Commit: one workgroup per request and kHold planes; rows of all heads lie side
// by side, and a lane holds one piece of a row in every plane.
__global__ void __launch_bounds__(kWg) kvx_commit_kernel(const CommitArgs a)
{
    __shared__ int64_t s_src[kWg], s_dst[kWg];
    const int tid = int(threadIdx.x), lane = tid & 63, R = a.c.num_requests;
    const int r = int(blockIdx.x) % R, plane0 = int(blockIdx.x) / R * kHold;
    const int planes = min(kHold, 2 * a.num_layers - plane0);
    // the path's length: entries ascend strictly and their slots lie in the row
    const int first = max(a.contexts[r], 0);
    const int32_t* const index = a.accepted + int64_t(r) * a.a_stride;
    const int most = min(a.counts[r], a.a_stride);
    int rows = 0;
    while (rows < most) {
        const int i = rows + lane;
        const int e = i < most ? index[i] : 0, before = i > 0 && i < most ? index[i - 1] : -1;
        const uint64_t good = __ballot(i < most && e > before && int64_t(first) + e < a.c.row_slots);
        if (good != ~uint64_t(0)) {
            rows += __builtin_ctzll(~good);
            break;
        }
        rows += 64;
    }
    if (plane0 == 0 && tid == 0) a.new_lens[r] = first + rows;
    if (planes <= 0) return;
    char* const base = a.c.base + plane0 * a.c.plane_bytes;
    float* const scales = a.c.scales ? a.c.scales + plane0 * a.c.plane_scales : nullptr;
    const int pieces = a.c.hd * a.c.row_bytes >> 4, lg = a.lg_lanes;
    const int per = 1 << lg, sets = kWg >> lg, set = tid >> lg, piece0 = tid & (per - 1);
    for (int i0 = 0; i0 < rows; i0 += kWg) {
        __syncthreads();                         // the last ones' places are read
        if (i0 + tid < rows) {
            const int i = i0 + tid, from = index[i];
            int64_t src = -1, dst = -1;
            if (from > i) {
                src = slot_row(a.c, r, first + from);
                dst = slot_row(a.c, r, first + i);
            }
            s_src[tid] = src < 0 || dst < 0 ? 0 : src;
            s_dst[tid] = src < 0 || dst < 0 ? -1 : dst;
        }
        __syncthreads();
        const int end = min(rows - i0, kWg);
        for (int row0 = 0; row0 < end; row0 += sets) {
            const int row = min(row0 + set, end - 1);
            const int64_t src = s_src[row], dst = row0 + set < end ? s_dst[row] : -1;
            for (int turn = 0; turn < pieces; turn += per) {
                const int piece = turn + piece0, part = min(piece, pieces - 1), head = min(piece, a.c.hd - 1);
                Held v;
#pragma unroll
                for (int k = 0; k < kHold; ++k) {
                    const int64_t p = min(k, planes - 1);
                    v.x[k] = *reinterpret_cast<const piece_t*>(base + p * a.c.plane_bytes +
                                                               src * a.c.row_bytes + part * 16);
                    v.s[k] = scales ? scales[p * a.c.plane_scales + src + head] : 0.0f;
                }
                arrived(v);
                __syncthreads();
#pragma unroll
                for (int k = 0; k < kHold; ++k)
                    if (k < planes && dst >= 0) {
                        if (piece < pieces)
                            *reinterpret_cast<piece_t*>(base + k * a.c.plane_bytes + dst * a.c.row_bytes + piece * 16) = v.x[k];
                        if (scales && piece < a.c.hd) scales[k * a.c.plane_scales + dst + piece] = v.s[k];
                    }
            }
        }
    }
}

template <bool kBf16, int kCache, int kPairing>
int append_by(const AppendArgs& a, void* stream)
{
    return launch_kernel(kvx_append_kernel<kBf16, kCache, kPairing>, a.b.total_tokens, kWg, stream, a);
}

template <bool kBf16, int kCache>
int append_to(const AppendArgs& a, void* stream)
{
    if (a.interleaved) return append_by<kBf16, kCache, kInterleaved>(a, stream);
    return a.pairs % 8 ? append_by<kBf16, kCache, kAnyHalves>(a, stream)
                       : append_by<kBf16, kCache, kHalves>(a, stream);
}

template <bool kBf16>
int append_as(const AppendArgs& a, int cache_dtype, void* stream)
{
    switch (cache_dtype) {
    case KVX_FP16: return append_to<kBf16, KVX_FP16>(a, stream);
    case KVX_BF16: return append_to<kBf16, KVX_BF16>(a, stream);
    case KVX_FP8_E4M3FN: return append_to<kBf16, KVX_FP8_E4M3FN>(a, stream);
    default: return append_to<kBf16, KVX_FP8_E5M2>(a, stream);
    }
}

// lanes of a row of `bytes`: 16 bytes each, a power of two, at most a workgroup's
int row_lanes(int64_t bytes)
{
    int lg = 0;
    while (lg < 8 && (int64_t(16) << lg) < bytes) ++lg;
    return lg;
}

// long requests take more threads, the passes over the weights being a chain (16001 slots, 32
// layers, the same buffers in every call: 119 us, 143 with 256 threads); short ones do not fill them (1100..1160 slots, 24
// requests in 4 layers: 90 us, 107 with 1024 threads)
int select_threads(int max_len) { return max_len > 4096 ? 1024 : kWg; }

// workgroups of a commit: at least one plane's, which write new_lens
int64_t commit_groups(const CacheArgs& c, int num_layers)
{
    return std::max<int64_t>(1, (2 * int64_t(num_layers) + kHold - 1) / kHold) * c.num_requests;
}

}  // namespace

double append_threads(int32_t tokens) { return double(tokens) * kWg; }

double evict_threads(const CacheArgs& c, int num_layers, int max_len)
{
    return double(num_layers) * c.num_requests * c.hd * std::max(select_threads(max_len), 2 * kWg);
}

double commit_threads(const CacheArgs& c, int num_layers) { return double(commit_groups(c, num_layers)) * kWg; }

int launch_append(const AppendArgs& a, int dtype, int cache_dtype, void* stream)
{
    return dtype == KVX_BF16 ? append_as<true>(a, cache_dtype, stream)
                             : append_as<false>(a, cache_dtype, stream);
}

int launch_evict(const EvictArgs& a, int num_layers, void* stream)
{
    const int64_t units = int64_t(num_layers) * a.c.num_requests * a.c.hd;
    const int err = select_threads(a.max_len) == 1024 ? launch_kernel(kvx_select_kernel<1024>, units, 1024, stream, a)
                                                      : launch_kernel(kvx_select_kernel<kWg>, units, kWg, stream, a);
    if (err) return err;
    MoveArgs m = {};
    m.c = a.c;
    m.kept = a.kept;
    m.budget = a.budget;
    m.lg_lanes = row_lanes(a.c.row_bytes);
    m.lens = a.lens;
    m.max_len = a.max_len;
    return a.c.row_bytes % 256 ? launch_kernel(kvx_move_kernel<false>, 2 * units, kWg, stream, m)
                               : launch_kernel(kvx_move_kernel<true>, 2 * units, kWg, stream, m);
}

int launch_commit(const CommitArgs& given, void* stream)
{
    CommitArgs a = given;
    a.lg_lanes = row_lanes(int64_t(a.c.hd) * a.c.row_bytes);
    return launch_kernel(kvx_commit_kernel, commit_groups(a.c, a.num_layers), kWg, stream, a);
}

}  // namespace kvx
