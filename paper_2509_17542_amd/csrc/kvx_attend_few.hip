// Attention of few query rows per KV head (one token, small trees) over the
// paged cache: up to 16 or 32 rows, the tokens of a request times the query
// heads of a KV head.
//
// Bound by reading K and V once.  A workgroup takes `chunk` slots of one request
// and KV head; its 4 waves take 32 slots at a time in turn, each with all the
// rows, and K and V go from memory to the matrix instructions' registers with no
// stop in LDS:
//   S^T = K Q^T   lane (slot, g) holds 8 elements of its slot's row: 16 bytes;
//   O^T = V^T P^T lane (m, g) holds, for 8 slots, the DT elements m DT .. of the
//                 row, so that 16 lanes read a row whole; element t of each is
//                 the operand of the t-th product, whose 16 result rows are
//                 the elements m DT + t.  The 8 slots are the ones whose
//                 weights the lane holds, so neither P nor V crosses lanes; V's
//                 16-bit pairs are put together by v_perm_b32.
// Where a slot's row lies is looked up once per chunk into LDS.
//
// 64 requests of 512..8192 slots, one token each (8 KV heads, 128 elements, bf16,
// 1.1 GB) take 214 us, 5.1 TB/s, and 5 for the join; one token over 255 slots 5.7.
// A plain stream of 256-byte pieces at 2 KB strides reads 6.4 TB/s, so what is left
// is the chunks' ends: places looked up before the first row, sums written after
// the last, and idle chunks of requests shorter than the longest.
// For the product with V a weight (8-bit codes: times its slot's scale) is taken as two
// 16-bit terms, itself rounded and what that left: the reads hide the second product
// (the calls above: 218.5 us with it and without; over an fp8 cache 154, 153; 256
// elements 326, 323).  With 17 to 32 rows it is one term, half a unit in the last
// place of its own, as in the many-rows kernel, which some of those calls take (trees of
// 8 nodes over an fp8 cache: 217 us with two, 209).  The sum of weights that divides
// is kept in fp32, as all sums are.
#include <hip/hip_runtime.h>

#include "kvx_attend_dev.h"

namespace kvx {
namespace {

constexpr int kWaves = 4;
constexpr int kWg = 64 * kWaves;
constexpr int kTile = 32;           // slots of a wave's turn
constexpr int kMaxChunk = 512;

template <int kBytes>
struct Words {
    uint32_t w[kBytes / 4];
};

// Rows that are read once: non-temporal (a stream of 256-byte pieces at strides of
// 2 KB reads at 6.5 TB/s so, at 5.8 without).
template <int kBytes>
__device__ __forceinline__ Words<kBytes> load_words(const char* p)
{
    constexpr int kN = kBytes / 4 < 4 ? kBytes / 4 : 4;
    typedef uint32_t part_t __attribute__((ext_vector_type(kN)));
    Words<kBytes> v;
#pragma unroll
    for (int i = 0; i < kBytes / 4 / kN; ++i) {
        const part_t x = __builtin_nontemporal_load(reinterpret_cast<const part_t*>(p) + i);
        if constexpr (kN == 1) {
            v.w[0] = __builtin_bit_cast(uint32_t, x);
        } else {
#pragma unroll
            for (int k = 0; k < kN; ++k) v.w[kN * i + k] = x[k];
        }
    }
    return v;
}

template <int kBytes>
__device__ __forceinline__ Words<kBytes> no_words()
{
    Words<kBytes> v;
#pragma unroll
    for (int i = 0; i < kBytes / 4; ++i) v.w[i] = 0;
    return v;
}

// One wave's tile: K as it is read, V as the matrix instructions take it.
template <int kCodes, int DP>
struct Tile {
    static constexpr int kEl = kCodes == kCodes16 ? 2 : 1;
    static constexpr int DT = DP / 16;
    static constexpr int kVBytes = DT * kEl;
    static constexpr int kRow = DP * kEl;           // bytes of a row
    static constexpr int kPieces = kRow / 16;       // 16-byte pieces of it, 8 elements or 16 codes
    static constexpr int kLoads = kTile * kRow / 1024;
    // Piece p of slot s lies at place p ^ turn_of(s) of the slot's row in LDS: 16 slots' pieces
    // of one number, which the matrix instructions take together, then lie in different banks.
    __device__ static __forceinline__ int turn_of(int s)
    {
        return kRow >= 256 ? s & 15 : (s / (256 / kRow)) & (kPieces - 1);
    }
    Words<16> k[kLoads];
    Words<kVBytes> v[8];
};

// Registers decide how many waves a SIMD holds: O takes DP RT / 4, K and V up to
// DP / 4 each.
template <int kCodes, int DP, int RT>
constexpr int kWavesPerSimd = DP >= 256 ? 1 : DP * RT >= 256 || (DP >= 128 && kCodes == kCodes16) ? 2 : 3;

template <bool kBf16, int kCodes, int DP, int RT, int kScores>
__global__ void __launch_bounds__(kWg, (kWavesPerSimd<kCodes, DP, RT>)) kvx_attend_few_kernel(const AttendArgs a)
{
    using T = Tile<kCodes, DP>;
    constexpr int DT = T::DT, kRows = 16 * RT;
    constexpr bool k8 = kCodes != kCodes16;
    constexpr bool kTwoTerms = RT == 1;
    constexpr bool kLift = k8 && !kBf16;
    constexpr float kUp = kLift ? kShift<kBf16> - kLiftShift : kShift<kBf16>;
    constexpr int kKeyBytes = kMaxChunk * (k8 ? 20 : 12);
    constexpr int kSlabBytes = 2 * kRows * DP * 4;
    __shared__ __attribute__((aligned(16))) char smem[kKeyBytes > kSlabBytes ? kKeyBytes : kSlabBytes];
    __shared__ __attribute__((aligned(16))) char s_k[kWaves][kTile * T::kRow];
    __shared__ uint64_t s_valid[kMaxChunk / 64];
    __shared__ float s_ml[kWaves][kRows][2];
    int64_t* const s_off = reinterpret_cast<int64_t*>(smem);
    int32_t* const s_pos = reinterpret_cast<int32_t*>(smem + kMaxChunk * 8);
    float* const s_ks = reinterpret_cast<float*>(smem + kMaxChunk * 12);
    float* const s_vs = reinterpret_cast<float*>(smem + kMaxChunk * 16);

    const int tid = int(threadIdx.x), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n16 = lane & 15, g = lane >> 4;
    const int D = a.c.dim, G = a.group;
    uint32_t u = blockIdx.x;
    const int h = int(u % uint32_t(a.c.hd));
    u /= uint32_t(a.c.hd);
    const int split = int(u % uint32_t(a.splits)), r = int(u / uint32_t(a.splits));
    const Request rq = request_of(a.c, a.b, r);
    const int rows = rq.n * G;
    if (rows == 0) return;
    const Range rg = range_of(a, rq, r, 0, rq.n - 1);
    const int v0 = split * a.chunk, v1 = min(v0 + a.chunk, rg.len);
    float* const part_ml = a.part_ml + int64_t(split) * a.b.total_tokens * a.q_heads * 2;
    if (a.splits > 1 && v0 >= v1) {
        for (int i = tid; i < rows; i += kWg) {
            const int tok = int(fast_div(uint32_t(i), a.div_group));
            const int64_t at = int64_t(rq.first + tok) * a.q_heads + h * G + (i - tok * G);
            part_ml[2 * at] = -INFINITY;
            part_ml[2 * at + 1] = 0.0f;
        }
        return;
    }

    // places of the chunk's slots
    for (int base = v0; base < v1; base += kWg) {
        const int v = base + tid, j = rg.slot(v);
        const int64_t row = v < v1 && j < rq.total ? slot_row(a.c, r, j) : -1;
        const uint64_t some = __ballot(row >= 0);
        if (lane == 0) s_valid[(v - v0) >> 6] = some;
        s_off[v - v0] = row < 0 ? 0 : (row + h) * a.c.row_bytes;
        s_pos[v - v0] = a.b.positions && j >= rq.ctx && j < rq.total ? a.b.positions[rq.first + j - rq.ctx] : j;
        if constexpr (k8) {
            s_ks[v - v0] = row < 0 ? 0.0f : a.c.scales[row + h];
            s_vs[v - v0] = row < 0 ? 0.0f : a.c.scales[a.c.plane_scales + row + h];
        }
    }

    // queries: rows n16 of each tile of 16, in the element order of K's pieces
    u32x4 q[RT][DP / 32];
    int tok[RT], qpos[RT];
    float slope2[RT];
    bool live[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int row = rt * 16 + n16;
        live[rt] = row < rows;
        const int rr = live[rt] ? row : 0;
        tok[rt] = int(fast_div(uint32_t(rr), a.div_group));
        const int head = h * G + (rr - tok[rt] * G);
        qpos[rt] = a.b.positions ? a.b.positions[rq.first + tok[rt]] : rq.ctx + tok[rt];
        slope2[rt] = a.slopes ? a.slopes[head] * kLog2e : 0.0f;
        const uint16_t* src = a.q + int64_t(rq.first + tok[rt]) * a.q_stride + int64_t(head) * D;
#pragma unroll
        for (int c = 0; c < DP / 32; ++c) {
            const int d = k8 ? (c >> 1) * 64 + g * 16 + (c & 1) * 8 : c * 32 + g * 8;
            q[rt][c] = u32x4{0, 0, 0, 0};
            if (live[rt] && d < D) q[rt][c] = *reinterpret_cast<const u32x4*>(src + d);
        }
    }
    const ScoreArgs sc = score_args(a);
    f32x4 o[RT][DT];
    float m[RT], l[RT], lift[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        m[rt] = -INFINITY;
        l[rt] = 0.0f;
        lift[rt] = kLiftMax;
#pragma unroll
        for (int t = 0; t < DT; ++t) o[rt][t] = f32x4{0, 0, 0, 0};
    }
    __syncthreads();

    const char* const kb = a.c.base;
    const char* const vb = a.c.base + a.c.plane_bytes;

    // Loads take no branch: a slot that lies in no page reads the plane's first
    // row, a lane past the row's end its first piece.  What comes of the former is
    // masked (turn), of the latter multiplied by q's zeros or not written.
    const int v_at = n16 * T::kVBytes < a.c.row_bytes ? n16 * T::kVBytes : 0;
    const int v_more = v_at + 16 < a.c.row_bytes ? v_at + 16 : 0;   // the second piece of 32 bytes

    // K: whole rows, 1 KB an instruction
    auto load_k = [&](int v, T& x) {
#pragma unroll
        for (int i = 0; i < T::kLoads; ++i) {
            const int s = (i * 64 + lane) / T::kPieces, piece = (i * 64 + lane) % T::kPieces * 16;
            x.k[i] = load_words<16>(kb + s_off[v - v0 + s] + (piece < a.c.row_bytes ? piece : 0));
        }
    };
    auto put_k = [&](const T& x) {
#pragma unroll
        for (int i = 0; i < T::kLoads; ++i) {
            const int s = (i * 64 + lane) / T::kPieces, place = ((i * 64 + lane) % T::kPieces) ^ T::turn_of(s);
            *reinterpret_cast<u32x4*>(s_k[wave] + s * T::kRow + place * 16) =
                u32x4{x.k[i].w[0], x.k[i].w[1], x.k[i].w[2], x.k[i].w[3]};
        }
    };
    // piece p of slot n16 of a half
    auto k_piece = [&](int half, int p) {
        const int s = 16 * half + n16;
        return *reinterpret_cast<const u32x4*>(s_k[wave] + s * T::kRow + ((p ^ T::turn_of(s)) << 4));
    };
    auto load_v = [&](int v, T& x) {   // slots 4 g .. 4 g + 3 of each half, elements n16 DT ..
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const char* const row = vb + s_off[v - v0 + 16 * (j >> 2) + 4 * g + (j & 3)];
            if constexpr (T::kVBytes == 32) {
                const Words<16> y = load_words<16>(row + v_at), z = load_words<16>(row + v_more);
#pragma unroll
                for (int i = 0; i < 4; ++i) x.v[j].w[i] = y.w[i], x.v[j].w[4 + i] = z.w[i];
            } else {
                x.v[j] = load_words<T::kVBytes>(row + v_at);
            }
        }
    };

    // the t-th operand of O^T = V^T P^T
    auto v_operand = [&](const T& x, int t) {
        u32x4 f;
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            if constexpr (!k8) {
                const uint32_t a0 = x.v[2 * p].w[t >> 1], a1 = x.v[2 * p + 1].w[t >> 1];
                f[p] = t & 1 ? pair16<true>(a0, a1) : pair16<false>(a0, a1);
            } else {
                const uint32_t a0 = x.v[2 * p].w[t >> 2], a1 = x.v[2 * p + 1].w[t >> 2];
                const uint32_t y = __builtin_amdgcn_perm(a1, a0, t & 2 ? 0x07030602u : 0x05010400u);
                f[p] = t & 1 ? widen2<kBf16, kCodes, true>(y) : widen2<kBf16, kCodes, false>(y);
            }
        }
        return f;
    };

    // the tile's slots that lie in a page
    auto valid_of = [&](int v) {
        return uint32_t(__builtin_amdgcn_readfirstlane(
            int(uint32_t(s_valid[(v - v0) >> 6] >> ((v - v0) & 32)))));
    };
    // whether every row sees the tile whole
    auto is_whole = [&](int v, uint32_t valid) {
        const int j0 = rg.slot(v);
        return j0 >= rg.all_lo && j0 + kTile <= rg.all_hi && valid == ~0u;
    };
    // what row tile rt sees of it, bit 16 e + i: slot 16 e + 4 g + i
    auto seen_by = [&](int rt, int v, uint32_t valid) {
        const uint64_t m = live[rt] ? seen_of(a, rq, r, tok[rt], qpos[rt], rg.slot(v), valid) : 0;
        return uint32_t(m) >> (4 * g);
    };
    // V's slots that lie in no page were read from another
    auto drop_v = [&](T& x, uint32_t valid) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (!(valid >> (4 * g) >> (16 * (j >> 2) + (j & 3)) & 1u)) x.v[j] = no_words<T::kVBytes>();
    };
    bool special = false;

    auto turn = [&](int v, int next, T& x) {
        const int at = v - v0;
        const uint32_t valid = valid_of(v);
        const bool whole = is_whole(v, valid);
        float ks[2][4], vs[2][4];
        if constexpr (k8) {
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    ks[s][i] = s_ks[at + 16 * s + 4 * g + i];
                    vs[s][i] = s_vs[at + 16 * s + 4 * g + i];
                }
        }
        put_k(x);
        load_k(next, x);               // the next turn's keys take their place
        f32x4 s[RT][2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) s[rt][e] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < DP / 32; ++c) {
                u32x4 f;
                if constexpr (k8) {
                    const u32x4 w = k_piece(e, 4 * (c >> 1) + g);
                    f = c & 1 ? widen8<kBf16, kCodes>(w.z, w.w) : widen8<kBf16, kCodes>(w.x, w.y);
                } else {
                    f = k_piece(e, 4 * c + g);
                }
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) s[rt][e] = mfma16<kBf16>(f, q[rt][c], s[rt][e]);
            }
        }
        u32x4 pf[RT], rest[kTwoTerms ? RT : 1];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            float y[2][4], top = -INFINITY;
            if constexpr (kScores == kPlain) {
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        y[e][i] = k8 ? s[rt][e][i] * (ks[e][i] * sc.c2) : s[rt][e][i] * sc.c2;
            } else {
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        y[e][i] = general_score<kScores>(sc, k8 ? s[rt][e][i] * ks[e][i] : s[rt][e][i], slope2[rt],
                                                         qpos[rt] - s_pos[at + 16 * e + 4 * g + i]);
            }
            uint32_t mine = ~0u;
            if (!whole) {
                mine = seen_by(rt, v, valid);
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!(mine >> (16 * e + i) & 1u)) y[e][i] = -INFINITY;
            }
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int i = 0; i < 4; ++i) top = fmaxf(top, y[e][i]);
            if (__any(top > m[rt] + kSlack)) {
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                const float to = fmaxf(m[rt], top);
                float alpha = to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m[rt] - to);
                l[rt] *= alpha;
                if constexpr (kLift) {
                    const float up = to == -INFINITY ? lift[rt] : fminf(lift[rt] + (to - m[rt]), kLiftMax);
                    if (to != -INFINITY) alpha = __builtin_amdgcn_exp2f((m[rt] - to) + (up - lift[rt]));
                    lift[rt] = up;
                }
                m[rt] = to;
#pragma unroll
                for (int t = 0; t < DT; ++t) o[rt][t] *= alpha;
            }
            const float base = (m[rt] == -INFINITY ? 0.0f : m[rt]) - kUp;
            float p[2][4];
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    p[e][i] = __builtin_amdgcn_exp2f(y[e][i] - base);
                    l[rt] += p[e][i];
                    if constexpr (k8) p[e][i] *= vs[e][i];
                }
            if (k8 && !whole) {
                // a scale of a slot that is not seen may be anything
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!(mine >> (16 * e + i) & 1u)) p[e][i] = 0.0f;
            }
            if constexpr (kLift) {
                float most = 0.0f;
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int i = 0; i < 4; ++i) most = fmaxf(most, finite_size(p[e][i]));
                if (__any(most * __builtin_amdgcn_exp2f(lift[rt]) > 32768.0f)) {   // 2^kLiftMost
                    most = fmaxf(most, __shfl_xor(most, 16));
                    most = fmaxf(most, __shfl_xor(most, 32));
                    const float to = lift_of(lift[rt], most), by = __builtin_amdgcn_exp2f(to - lift[rt]);
                    lift[rt] = to;
#pragma unroll
                    for (int t = 0; t < DT; ++t) o[rt][t] *= by;
                }
                const float by = __builtin_amdgcn_exp2f(lift[rt]);
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int i = 0; i < 4; ++i) p[e][i] *= by;
            }
            pf[rt] = u32x4{pack2<kBf16>(p[0][0], p[0][1]), pack2<kBf16>(p[0][2], p[0][3]),
                           pack2<kBf16>(p[1][0], p[1][1]), pack2<kBf16>(p[1][2], p[1][3])};
            if constexpr (kTwoTerms)
#pragma unroll
                for (int w = 0; w < 4; ++w)
                    rest[rt][w] = pack2<kBf16>(p[w >> 1][2 * (w & 1)] - value16<kBf16>(pf[rt][w] & 0xFFFFu),
                                               p[w >> 1][2 * (w & 1) + 1] - value16<kBf16>(pf[rt][w] >> 16));
        }
        if (!whole) {
            drop_v(x, valid);
            uint32_t found = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int i = 0; i < T::kVBytes / 4; ++i) {
                    const uint32_t f = nonfinite<kBf16, kCodes>(x.v[j].w[i]);
                    x.v[j].w[i] = without<kCodes>(x.v[j].w[i], f);
                    found |= f;
                }
            special |= __any(found != 0) != 0;
        }
#pragma unroll
        for (int t = 0; t < DT; ++t) {
            const u32x4 f = v_operand(x, t);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                o[rt][t] = mfma16<kBf16>(f, pf[rt], o[rt][t]);
                if constexpr (kTwoTerms) o[rt][t] = mfma16<kBf16>(f, rest[rt], o[rt][t]);
            }
        }
    };

    int v = v0 + wave * kTile;
    if (v < v1) {
        T x;
        load_k(v, x);
        for (; v < v1; v += kWaves * kTile) {
            load_v(v, x);
            turn(v, v + kWaves * kTile < v1 ? v + kWaves * kTile : v, x);
        }
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) special |= __any(live[rt] && any_endless<4, DT>(o[rt])) != 0;
    if (__builtin_expect(special, 0)) {
        // the tiles again, an element of V's rows at a time: which sums had infinities or NaN
        const int place = hidden(lane), n16 = place & 15, g = place >> 4;
        Had<4 * DT> had[RT];
#pragma unroll 1
        for (v = v0 + wave * kTile; v < v1; v += kWaves * kTile) {
            const uint32_t valid = valid_of(v);
#pragma unroll 1
            for (int t = 0; t < DT; ++t) {
                const int byte = (n16 * DT + t) * T::kEl, at = byte < a.c.row_bytes ? byte : 0;
                u32x4 f = {0, 0, 0, 0};
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int slot = 16 * (j >> 2) + 4 * g + (j & 3);
                    const char* const from = vb + s_off[v - v0 + slot] + at;
                    uint32_t x;
                    if constexpr (k8)
                        x = times2<kBf16>(widen2<kBf16, kCodes, false>(*reinterpret_cast<const uint8_t*>(from)),
                                          scale_kind(s_vs[v - v0 + slot]), 0.0f) & 0xFFFFu;
                    else
                        x = *reinterpret_cast<const uint16_t*>(from);
                    f[j >> 1] |= (valid >> slot & 1u ? x : 0u) << (16 * (j & 1));
                }
                uint32_t some = 0;
#pragma unroll
                for (int p = 0; p < 4; ++p) some |= nonfinite<kBf16, kCodes16>(f[p]);
                if (!__any(some != 0)) continue;
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    const int row = rt * 16 + n16, i = int(fast_div(uint32_t(row < rows ? row : 0), a.div_group));
                    const int pos = a.b.positions ? a.b.positions[rq.first + i] : rq.ctx + i;
                    const uint32_t mine =
                        row < rows ? uint32_t(seen_of(a, rq, r, i, pos, rg.slot(v), valid)) >> (4 * g) : 0u;
                    u32x4 seen;
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const uint32_t two = mine >> (16 * (w >> 1) + 2 * (w & 1)) & 3u;
                        seen[w] = (two & 1u ? kOne<kBf16> : 0u) | (two & 2u ? kOne<kBf16> << 16 : 0u);
                    }
#pragma unroll
                    for (int kind = 1; kind <= 3; ++kind) {
                        const f32x4 count = mfma16<kBf16>(classify8<kBf16>(f, kind), seen, f32x4{0, 0, 0, 0});
#pragma unroll
                        for (int i = 0; i < 4; ++i) had[rt].add(4 * t + i, count[i], kind);
                    }
                }
            }
        }
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[rt][t][i] = had[rt].of(4 * t + i, o[rt][t][i]);
    }

    // the waves' sums, joined through LDS two at a time
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        l[rt] += __shfl_xor(l[rt], 16);
        l[rt] += __shfl_xor(l[rt], 32);
        if constexpr (kLift) l[rt] *= 65536.0f;          // 2^kLiftShift
        m[rt] = reference_of(m[rt], l[rt]);
        if (g == 0) {
            s_ml[wave][rt * 16 + n16][0] = m[rt];
            s_ml[wave][rt * 16 + n16][1] = l[rt];
        }
    }
    __syncthreads();
    float* const slab = reinterpret_cast<float*>(smem) + (wave & 1) * kRows * DP;
    float scale[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) top = fmaxf(top, s_ml[w][rt * 16 + n16][0]);
        scale[rt] = m[rt] == -INFINITY ? 0.0f
                    : kLift            ? unlifted(lift[rt], m[rt] - top)
                                       : __builtin_amdgcn_exp2f(m[rt] - top);
    }
    if (__builtin_expect(special, 0)) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[rt][t][i] = weighted(o[rt][t][i], scale[rt]);
            scale[rt] = 1.0f;
        }
    }
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        if ((wave >> 1) == half) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int t = 0; t < DT; ++t) {
                        float* const at = slab + (rt * 16 + n16) * DP + (4 * g + i) * DT + t;
                        const float x = o[rt][t][i] * scale[rt];
                        *at = half == 0 ? x : *at + x;
                    }
        }
        __syncthreads();
    }
    const float* const sum = reinterpret_cast<const float*>(smem);
    for (int i = tid; i < rows * (DP / 8); i += kWg) {
        const int row = i / (DP / 8), d = i % (DP / 8) * 8;
        if (d >= D) continue;
        float top = -INFINITY, total = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) top = fmaxf(top, s_ml[w][row][0]);
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
            total += s_ml[w][row][0] == -INFINITY ? 0.0f
                                                  : s_ml[w][row][1] * __builtin_amdgcn_exp2f(s_ml[w][row][0] - top);
        const int t = int(fast_div(uint32_t(row), a.div_group));
        const int64_t token = rq.first + t, head = h * G + (row - t * G);
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = sum[row * DP + d + e] + sum[kRows * DP + row * DP + d + e];
        if (a.splits > 1) {
            const int64_t at = token * a.q_heads + head;
            float4* const out = reinterpret_cast<float4*>(
                a.part_o + (int64_t(split) * a.b.total_tokens * a.q_heads + at) * D + d);
            out[0] = make_float4(x[0], x[1], x[2], x[3]);
            out[1] = make_float4(x[4], x[5], x[6], x[7]);
            if (d == 0) {
                part_ml[2 * at] = reference_of(top, total);
                part_ml[2 * at + 1] = total;
            }
        } else {
            const float inv = total == 0.0f ? 0.0f : 1.0f / total;
            u32x4 w;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                w[e] = total == 0.0f ? 0u : pack2<kBf16>(x[2 * e] * inv, x[2 * e + 1] * inv);
            *reinterpret_cast<u32x4*>(a.out + token * a.out_stride + head * D + d) = w;
            if (a.lse && d == 0)
                a.lse[token * a.q_heads + head] =
                    total == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(total) - kShift<kBf16>) * kLn2;
        }
    }
}

template <bool kBf16, int kCodes, int DP, int RT, int kScores>
int go_as(const AttendArgs& a, void* stream)
{
    return launch_kernel(kvx_attend_few_kernel<kBf16, kCodes, DP, RT, kScores>,
                         int64_t(a.c.num_requests) * a.splits * a.c.hd, kWg, stream, a);
}

template <bool kBf16, int kCodes, int DP, int RT>
int go(const AttendArgs& a, void* stream)
{
    switch (scores_of(a)) {
    case kWide: return go_as<kBf16, kCodes, DP, RT, kWide>(a, stream);
    case kGeneral: return go_as<kBf16, kCodes, DP, RT, kGeneral>(a, stream);
    default: return go_as<kBf16, kCodes, DP, RT, kPlain>(a, stream);
    }
}

template <bool kBf16, int kCodes>
int pick(const AttendArgs& a, const AttendPlan& p, void* stream)
{
    const bool two = p.tile_rows > 16;
    if (a.c.dim <= 64) return two ? go<kBf16, kCodes, 64, 2>(a, stream) : go<kBf16, kCodes, 64, 1>(a, stream);
    if (a.c.dim <= 128) return two ? go<kBf16, kCodes, 128, 2>(a, stream) : go<kBf16, kCodes, 128, 1>(a, stream);
    return go<kBf16, kCodes, 256, 1>(a, stream);
}

}  // namespace

int launch_few(const AttendArgs& a, const AttendPlan& p, int dtype, int cache_dtype, void* stream)
{
    const bool bf = dtype == KVX_BF16;
    switch (cache_dtype) {
    case KVX_FP8_E4M3FN: return bf ? pick<true, kCodesE4m3>(a, p, stream) : pick<false, kCodesE4m3>(a, p, stream);
    case KVX_FP8_E5M2: return bf ? pick<true, kCodesE5m2>(a, p, stream) : pick<false, kCodesE5m2>(a, p, stream);
    default: return bf ? pick<true, kCodes16>(a, p, stream) : pick<false, kCodes16>(a, p, stream);
    }
}

}  // namespace kvx
