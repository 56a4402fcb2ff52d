// Attention of many query rows per KV head (wide trees, chains) over the paged
// cache; each type of cache is a source of its own (kvx_attend_rows_*.hip), which
// includes this one.
//
// A workgroup takes 32 rows per wave (rows are tokens times the query heads of
// a KV head, tokens outermost) of one request and KV head, and walks the
// slots that they see, KT at a time through LDS: K as rows, V transposed, both
// widened to the queries' type and padded so that 16 lanes' 16-byte reads meet
// every bank once.  While one tile is used the next one's rows are on their
// way to registers, and the places of the one after that are looked up.
//   S^T = K Q^T: a lane holds, of its query row, slots 8 q + 4 h + (0..3) of each
//   32 (h: which half of the wave);
//   O^T = V^T P^T: the weights go on as they lie, 8 of a lane's as one operand;
//   V is laid out in LDS in that order of slots.
// Where the row tiles' workgroups (requests x splits x KV heads) are a multiple of 8,
// those that read the same slots are dealt to one XCD.
//
// Bound by the matrix instructions and the exponentials between them: 1024
// matrix cycles of a SIMD for a tile of 64 slots and 128 rows of 128 elements,
// 210 (plain scores) to 360 (capped, 8-bit codes) vector instructions, and the
// wait of one for the other; and by LDS, out of which each wave reads all of a tile:
// for chunks of many tokens it is busy 39% of the cycles (30% of these conflicts),
// the matrix pipes 32%.  8 requests of 2048 tokens on 8192 slots run at 807 to 835
// TFLOP/s in fp16 and 850 in bf16 (a library's large product of that type alone:
// 1342, 1410); three chunks of 1024..2048 tokens with a bias, a window and a
// prefix, whose edges cost partial tiles, in 0.64 to 0.69 ms, 730 to 780 TFLOP/s; 16
// trees of 16..64 nodes over an fp8 cache of 2048..16384 slots, capped scores, in
// 318 to 325 us, 24 of them the join.  These are times of a card in use: its first
// milliseconds of such work after a pause run at about 2 GHz, not 2.4 (0.72 ms and 380
// us).
//
// 128 rows share a tile, 64 slots of it; up to 64 rows have half the waves, so that
// none only stages, and 32 slots, so that twice as many workgroups fit a CU's LDS
// (trees of 9..16 nodes, 36..64 rows, over the same fp8 cache: 165 us, 190 in workgroups of
// 128; 64 such over a bf16 cache of 512..8192 slots 303, 340; in longer runs now 154 and 293).
// A weight (8-bit codes: times its slot's scale) goes to 16 bits for the product with
// V; its rounding is the type's own half unit in the last place, relative (a second
// product with what it left would cost the three chunks 816 us, 657 without, and the 16
// trees 365, 323), and the sum of weights that divides is kept in fp32.  Sums, references
// and outputs stay in fp32 until the end.
#pragma once

#include <hip/hip_runtime.h>

#include "kvx_attend_dev.h"

namespace kvx {
namespace {

// Here scores with a cap (and perhaps a bias) are kept apart from those with a bias
// alone (or another scale).
enum RowsScores : int { kBiased = kGeneral, kCappedWide = kWide, kCapped = 3 };

template <int kCodes, int DP, int NW>
struct Shape {
    static constexpr int kWg = 64 * NW;
    static constexpr int KT = DP >= 256 || NW == 2 ? 32 : 64; // slots of a tile
    static constexpr int kEl = kCodes == kCodes16 ? 2 : 1;
    static constexpr int kKRow = DP * 2 + 16;               // LDS bytes of a slot's K
    // LDS bytes of an element's V: KT / 8 pieces of 8 slots, piece g at place g ^ (d / 16 % 4),
    // so that neither the writes (a lane to every 4 elements) nor the reads meet in a bank
    static constexpr int kVRow = KT * 2 + 16;
    static constexpr int kKUnits = KT * DP / 8;             // 8 elements of a slot
    static constexpr int kVUnits = (KT / 8) * (DP / 4);     // 4 elements of 8 slots
    static constexpr int kKPer = (kKUnits + kWg - 1) / kWg;
    static constexpr int kVPer = (kVUnits + kWg - 1) / kWg;
    static constexpr int kBatch = kWg / KT;                 // tiles whose places are looked up at once
    static constexpr int kRing = 2 * kBatch;
};

template <bool kBf16, int kCodes, int DP, int NW, int kScores>
__global__ void __launch_bounds__(64 * NW, (DP >= 256 ? 1 : 2)) kvx_attend_rows_kernel(const AttendArgs a, int row_tiles)
{
    using S = Shape<kCodes, DP, NW>;
    constexpr int KT = S::KT, kWg = S::kWg, ST = KT / 32, DTB = DP / 32;
    constexpr bool k8 = kCodes != kCodes16;
    constexpr bool kLift = k8 && !kBf16;
    constexpr float kUp = kLift ? kShift<kBf16> - kLiftShift : kShift<kBf16>;
    constexpr uint64_t kAll = KT == 64 ? ~uint64_t(0) : (uint64_t(1) << (KT & 63)) - 1;
    __shared__ __attribute__((aligned(16))) char s_k[2][KT * S::kKRow];
    __shared__ __attribute__((aligned(16))) char s_v[2][DP * S::kVRow];
    __shared__ int64_t s_off[2 * kWg];
    __shared__ __attribute__((aligned(16))) float s_ks[k8 ? 2 * kWg : 1];
    __shared__ __attribute__((aligned(16))) float s_vs[k8 ? 2 * kWg : 1];
    __shared__ uint64_t s_valid[S::kRing];
    __shared__ int s_special;

    const int tid = int(threadIdx.x), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n32 = lane & 31, half = lane >> 5;
    const int D = a.c.dim, G = a.group;

    // the last rows, which see the most slots, first
    const uint32_t groups = uint32_t(a.c.num_requests) * uint32_t(a.splits) * uint32_t(a.c.hd);
    const uint32_t group = blockIdx.x % groups;
    const int rt = row_tiles - 1 - int(blockIdx.x / groups);
    uint32_t u = group;
    const int h = int(u % uint32_t(a.c.hd));
    u /= uint32_t(a.c.hd);
    const int split = int(u % uint32_t(a.splits)), r = int(u / uint32_t(a.splits));
    const Request rq = request_of(a.c, a.b, r);
    const int rows = rq.n * G, row0 = rt * 32 * NW;
    if (row0 >= rows) return;
    const int i0 = int(fast_div(uint32_t(row0), a.div_group));
    const int i1 = int(fast_div(uint32_t(min(row0 + 32 * NW, rows) - 1), a.div_group));
    const Range rg = range_of(a, rq, r, i0, i1);
    const int v0 = split * a.chunk, v1 = min(v0 + a.chunk, rg.len);
    const int tiles = v1 > v0 ? (v1 - v0 + KT - 1) / KT : 0;
    // The last slots first: with a bias by distance they weigh most, and the rows' references are
    // then hardly ever moved (chunks of 1024..2048 tokens with a bias: 860 us the other way
    // round, as against 717 without one).
    auto tile_at = [&](int t) { return v0 + (tiles - 1 - t) * KT; };

    const bool busy = row0 + wave * 32 < rows;   // the last workgroup's last waves may only stage
    // this lane's query row
    const int row = row0 + wave * 32 + n32;
    const bool live = row < rows;
    const int rr = live ? row : row0;
    const int tok = int(fast_div(uint32_t(rr), a.div_group)), head = h * G + (rr - tok * G);
    const int64_t token = rq.first + tok;
    const int qpos = a.b.positions ? a.b.positions[token] : rq.ctx + tok;
    const float slope2 = a.slopes ? a.slopes[head] * kLog2e : 0.0f;
    u32x4 q[DP / 16];
    {
        const uint16_t* const src = a.q + token * a.q_stride + int64_t(head) * D;
#pragma unroll
        for (int c = 0; c < DP / 16; ++c) {
            const int d = c * 16 + half * 8;
            q[c] = u32x4{0, 0, 0, 0};
            if (live && d < D) q[c] = *reinterpret_cast<const u32x4*>(src + d);
        }
    }
    const ScoreArgs sc = score_args(a);
    const float scale2 = kScores == kCapped ? sc.to_cap : sc.c2;
    f32x16 o[DTB];
#pragma unroll
    for (int t = 0; t < DTB; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] = 0.0f;
    float m = -INFINITY, l = 0.0f, lift = kLiftMax;

    const char* const kb = a.c.base;
    const char* const vb = a.c.base + a.c.plane_bytes;

    if (tid == 0) s_special = 0;

    // ---- places: a slot to each lane, kBatch tiles at a time ----
    // Looked up a batch ahead, noted at the start of the batch before their own;
    // 8-bit scales are read from there on and noted one tile later.  Ahead of its
    // barrier a tile's workgroup then knows where the next tile's rows lie.
    int64_t f_row = -1;
    float f_ks = 0.0f, f_vs = 0.0f;
    auto look_up = [&](int batch) {
        const int t = batch * S::kBatch + tid / KT, v = tile_at(t) + tid % KT, j = rg.slot(v);
        f_row = t < tiles && v < v1 && j < rq.total ? slot_row(a.c, r, j) : -1;
    };
    auto note_places = [&](int batch) {
        const int at = (batch & 1) * kWg + tid;
        const uint64_t valid = __ballot(f_row >= 0);
        if constexpr (KT == 64) {
            if (lane == 0) s_valid[at / KT] = valid;
        } else {
            if (n32 == 0) s_valid[at / KT] = uint32_t(valid >> (lane & 32));
        }
        s_off[at] = f_row < 0 ? 0 : (f_row + h) * a.c.row_bytes;
        if constexpr (k8) {
            f_ks = f_row < 0 ? 0.0f : a.c.scales[f_row + h];
            f_vs = f_row < 0 ? 0.0f : a.c.scales[a.c.plane_scales + f_row + h];
        }
    };
    auto note_scales = [&](int batch) {
        if constexpr (k8) {
            // a key's scale, times what products are scaled by anyway
            s_ks[(batch & 1) * kWg + tid] = f_ks * scale2;
            s_vs[(batch & 1) * kWg + tid] = f_vs;
        }
    };

    // ---- rows of a tile: memory -> registers -> LDS ----
    // A slot that lies in no page reads the plane's first row, a lane past the
    // row's end its first piece: what comes of the former is masked (store, use),
    // of the latter multiplied by q's zeros or not written.
    static_assert(S::kKUnits % kWg == 0 && kWg % (DP / 4) == 0, "a thread's pieces lie at one place of the rows");
    const int k_piece = tid % (DP / 8) * 8 * S::kEl, v_piece = tid % (DP / 4) * 4 * S::kEl;
    const char* const k_base = kb + (k_piece < a.c.row_bytes ? k_piece : 0);
    const char* const v_base = vb + (v_piece < a.c.row_bytes ? v_piece : 0);
    u32x4 kr[S::kKPer];
    uint2 vr[S::kVPer][8];
    int64_t k_off[S::kKPer], v_off[S::kVPer][8];
    auto places = [&](int t) {
        const int64_t* const off = s_off + (t & (S::kRing - 1)) * KT;
#pragma unroll
        for (int i = 0; i < S::kKPer; ++i) k_off[i] = off[(tid + i * kWg) / (DP / 8)];
#pragma unroll
        for (int i = 0; i < S::kVPer; ++i) {
            const int kg = min((tid + i * kWg) / (DP / 4), KT / 8 - 1), first = (kg >> 1) * 16 + (kg & 1) * 4;
#pragma unroll
            for (int e = 0; e < 8; ++e) v_off[i][e] = off[first + (e & 3) + (e >> 2) * 8];
        }
    };
    auto valid_of = [&](int t) {
        const uint64_t v = s_valid[t & (S::kRing - 1)];
        return uint64_t(uint32_t(__builtin_amdgcn_readfirstlane(int(uint32_t(v >> 32))))) << 32 |
               uint32_t(__builtin_amdgcn_readfirstlane(int(uint32_t(v))));
    };
    auto load = [&]() {
#pragma unroll
        for (int i = 0; i < S::kKPer; ++i) {
            const char* const p = k_base + k_off[i];
            if constexpr (k8) {
                const uint2 w = *reinterpret_cast<const uint2*>(p);
                kr[i].x = w.x, kr[i].y = w.y;
            } else {
                kr[i] = *reinterpret_cast<const u32x4*>(p);
            }
        }
#pragma unroll
        for (int i = 0; i < S::kVPer; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const char* const p = v_base + v_off[i][e];
                if constexpr (k8)
                    vr[i][e].x = *reinterpret_cast<const uint32_t*>(p);
                else
                    vr[i][e] = *reinterpret_cast<const uint2*>(p);
            }
    };
    auto whole_tile = [&](int t, uint64_t valid) {
        const int j0 = rg.slot(tile_at(t));
        return j0 >= rg.all_lo && j0 + KT <= rg.all_hi && valid == kAll;
    };
    // element e of 8 slots, in the queries' type
    auto column = [&](const uint2 (&x)[8], int e) {
        u32x4 w;
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            if constexpr (k8) {
                const uint32_t y = __builtin_amdgcn_perm(x[2 * p + 1].x, x[2 * p].x,
                                                         e & 2 ? 0x07030602u : 0x05010400u);
                w[p] = e & 1 ? widen2<kBf16, kCodes, true>(y) : widen2<kBf16, kCodes, false>(y);
            } else {
                const uint32_t y0 = e & 2 ? x[2 * p].y : x[2 * p].x;
                const uint32_t y1 = e & 2 ? x[2 * p + 1].y : x[2 * p + 1].x;
                w[p] = e & 1 ? pair16<true>(y0, y1) : pair16<false>(y0, y1);
            }
        }
        return w;
    };
    // K, and V with its values that are not finite as 0 where not every row sees the tile whole
    auto store = [&](int t, uint64_t valid) {
        char* const ks = s_k[t & 1];
        char* const vs = s_v[t & 1];
        const bool whole = whole_tile(t, valid);
#pragma unroll
        for (int i = 0; i < S::kKPer; ++i) {
            const int unit = tid + i * kWg;
            const int key = unit / (DP / 8), d = unit % (DP / 8) * 8;
            u32x4 w = kr[i];
            if constexpr (k8) w = widen8<kBf16, kCodes>(kr[i].x, kr[i].y);
            *reinterpret_cast<u32x4*>(ks + key * S::kKRow + d * 2) = w;
        }
#pragma unroll
        for (int i = 0; i < S::kVPer; ++i) {
            const int unit = tid + i * kWg;
            if (S::kVUnits % kWg && unit >= S::kVUnits) break;
            const int kg = unit / (DP / 4), d = unit % (DP / 4) * 4;
            char* const out = vs + d * S::kVRow + (kg ^ ((d >> 4) & 3)) * 16;
            if (whole) {
#pragma unroll
                for (int e = 0; e < 4; ++e) *reinterpret_cast<u32x4*>(out + e * S::kVRow) = column(vr[i], e);
            } else {
                const int first = (kg >> 1) * 16 + (kg & 1) * 4;
                uint32_t found = 0;
                uint2 x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    x[e] = valid >> (first + (e & 3) + (e >> 2) * 8) & 1 ? vr[i][e] : make_uint2(0, 0);
                    found |= nonfinite<kBf16, kCodes>(x[e].x);
                    if constexpr (!k8) found |= nonfinite<kBf16, kCodes>(x[e].y);
                }
                if (found) s_special = 1;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const u32x4 w = column(x, e);
                    *reinterpret_cast<u32x4*>(out + e * S::kVRow) = found ? classify8<kBf16>(w, 0) : w;
                    __builtin_amdgcn_sched_barrier(0);  // one at a time: this path is rare
                }
            }
        }
    };

    auto seen_by_me = [&](int t, uint64_t valid) {
        uint64_t mine = ~uint64_t(0);
        if (live) mine = seen_of(a, rq, r, tok, qpos, rg.slot(tile_at(t)), valid);
        return mine >> (4 * half);
    };
    auto use = [&](int t, uint64_t valid) {
        const int ring = t & (S::kRing - 1);
        const bool whole = whole_tile(t, valid);
        const char* const kl = s_k[t & 1] + n32 * S::kKRow + half * 16;
        const char* const vl = s_v[t & 1] + n32 * S::kVRow + (half ^ (n32 >> 4)) * 16;
        f32x16 s[ST];
#pragma unroll
        for (int e = 0; e < ST; ++e)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[e][i] = 0.0f;
#pragma unroll
        for (int c = 0; c < DP / 16; ++c)
#pragma unroll
            for (int e = 0; e < ST; ++e)
                s[e] = mfma32<kBf16>(*reinterpret_cast<const u32x4*>(kl + e * 32 * S::kKRow + c * 32), q[c], s[e]);
        // Scores relative to the row's reference so far; element i of s[e] is slot
        // 32 e + 8 (i / 4) + 4 half + i % 4.
        float base = (m == -INFINITY ? 0.0f : m) - kUp;
        float by = scale2;                       // what the products are still to be multiplied by
        if constexpr (k8) {
            by = 1.0f;
#pragma unroll
            for (int e = 0; e < ST; ++e)
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const int at = 32 * e + 8 * b + 4 * half;
                    const f32x4 ks = *reinterpret_cast<const f32x4*>(s_ks + ring * KT + at);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        s[e][4 * b + i] = kScores != kPlain ? s[e][4 * b + i] * ks[i]
                                                          : __builtin_fmaf(s[e][4 * b + i], ks[i], -base);
                }
        }
        if constexpr (kScores != kPlain) {
            const int j0 = rg.slot(tile_at(t));
            const bool in_order = !a.b.positions || j0 + KT <= rq.ctx;  // slot j lies at position j
            const bool linear = kScores == kBiased && in_order && __all(qpos - j0 >= KT);
            if constexpr (kScores == kCapped) {
#pragma unroll
                for (int e = 0; e < ST; ++e)
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[e][i] = capped(sc, s[e][i] * by, -base);
            } else if constexpr (kScores == kCappedWide) {
#pragma unroll
                for (int e = 0; e < ST; ++e)
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[e][i] = capped_wide(sc, s[e][i] * by, -base);
            } else if (linear) {
                // all slots before the token: linear in the slot
                const float first = slope2 * static_cast<float>(j0 + 4 * half - qpos) - base;
#pragma unroll
                for (int e = 0; e < ST; ++e)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        s[e][i] = __builtin_fmaf(s[e][i], by,
                                                 __builtin_fmaf(slope2, float(32 * e + 8 * (i >> 2) + (i & 3)), first));
            } else {
#pragma unroll
                for (int e = 0; e < ST; ++e)
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[e][i] = __builtin_fmaf(s[e][i], by, -base);
            }
            if (a.slopes && !linear) {
                if (in_order) {
                    const float ahead = static_cast<float>(qpos - j0 - 4 * half);
#pragma unroll
                    for (int e = 0; e < ST; ++e)
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            s[e][i] = __builtin_fmaf(-slope2,
                                                     __builtin_fabsf(ahead - float(32 * e + 8 * (i >> 2) + (i & 3))),
                                                     s[e][i]);
                } else {
#pragma unroll
                    for (int e = 0; e < ST; ++e)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int j = j0 + 32 * e + 8 * (i >> 2) + 4 * half + (i & 3);
                            const int distance = qpos - place_of(a, rq, j);
                            s[e][i] -= slope2 * static_cast<float>(distance < 0 ? -distance : distance);
                            __builtin_amdgcn_sched_barrier(0);  // one at a time: few tiles come here
                        }
                }
            }
        } else if constexpr (!k8) {
#pragma unroll
            for (int e = 0; e < ST; ++e)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[e][i] = __builtin_fmaf(s[e][i], by, -base);
        }
        uint64_t mine = ~uint64_t(0);
        if (!whole) {
            mine = seen_by_me(t, valid);
#pragma unroll
            for (int e = 0; e < ST; ++e)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (!(mine >> (32 * e + 8 * (i >> 2) + (i & 3)) & 1)) s[e][i] = -INFINITY;
        }
        float top = -INFINITY;
#pragma unroll
        for (int e = 0; e < ST; ++e)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[e][i]);
        if (__any(top > (m == -INFINITY ? -INFINITY : kSlack + kUp))) {
            top = fmaxf(top, __shfl_xor(top, 32));
            const float to = fmaxf(m, top + base);
            float alpha = to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - to);
            const float by2 = base - ((to == -INFINITY ? 0.0f : to) - kUp);
            l *= alpha;
            if constexpr (kLift) {
                const float up = to == -INFINITY ? lift : fminf(lift + (to - m), kLiftMax);
                if (to != -INFINITY) alpha = __builtin_amdgcn_exp2f((m - to) + (up - lift));
                lift = up;
            }
            m = to;
#pragma unroll
            for (int t2 = 0; t2 < DTB; ++t2) o[t2] *= alpha;
#pragma unroll
            for (int e = 0; e < ST; ++e)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[e][i] += by2;
        }
        // weights, times their slots' scales
        auto weights = [&](int e, int b, float (&p)[4]) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                p[i] = __builtin_amdgcn_exp2f(s[e][4 * b + i]);
                l += p[i];
            }
            if constexpr (k8) {
                const f32x4 vs = *reinterpret_cast<const f32x4*>(s_vs + ring * KT + 32 * e + 8 * b + 4 * half);
#pragma unroll
                for (int i = 0; i < 4; ++i) p[i] *= vs[i];
                if (!whole) {
                    // a scale of a slot that is not seen may be anything
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!(mine >> (32 * e + 8 * b + i) & 1)) p[i] = 0.0f;
                }
            }
        };
        float by_lift = 1.0f;
        if constexpr (kLift) {
            float most = 0.0f;
#pragma unroll
            for (int e = 0; e < ST; ++e)
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    float p[4];
                    weights(e, b, p);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        s[e][4 * b + i] = p[i];
                        most = fmaxf(most, finite_size(p[i]));
                    }
                }
            if (__any(most * __builtin_amdgcn_exp2f(lift) > 32768.0f)) {   // 2^kLiftMost
                const float to_lift = lift_of(lift, fmaxf(most, __shfl_xor(most, 32)));
                const float by_o = __builtin_amdgcn_exp2f(to_lift - lift);
                lift = to_lift;
#pragma unroll
                for (int t2 = 0; t2 < DTB; ++t2) o[t2] *= by_o;
            }
            by_lift = __builtin_amdgcn_exp2f(lift);
        }
        u32x4 pf[ST][2];
#pragma unroll
        for (int e = 0; e < ST; ++e)
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                float p[4];
                if constexpr (kLift) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) p[i] = s[e][4 * b + i] * by_lift;
                } else {
                    weights(e, b, p);
                }
                pf[e][b >> 1][2 * (b & 1)] = pack2<kBf16>(p[0], p[1]);
                pf[e][b >> 1][2 * (b & 1) + 1] = pack2<kBf16>(p[2], p[3]);
            }
#pragma unroll
        for (int e = 0; e < ST; ++e)
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int t2 = 0; t2 < DTB; ++t2)
                    o[t2] = mfma32<kBf16>(*reinterpret_cast<const u32x4*>(vl + t2 * 32 * S::kVRow + e * 64 + (b ^ (t2 & 1)) * 32),
                                          pf[e][b], o[t2]);
    };

    if (tiles > 0) {
        look_up(0);
        note_places(0);
        note_scales(0);
        look_up(1);
        __syncthreads();
        places(0);
        uint64_t valid = valid_of(0);
        load();
        for (int t = 0; t < tiles; ++t) {
            const int batch = t / S::kBatch, phase = t % S::kBatch;
            const int next = min(t + 1, tiles - 1);  // the last again: nothing waits for it
            store(t, valid);
            if (phase == 1) note_scales(batch + 1);
            places(next);
            const uint64_t next_valid = valid_of(next);
            if (phase == 0) note_places(batch + 1);
            __syncthreads();
            load();
            if (phase == 0) look_up(batch + 2);
            if (busy) use(t, valid);
            valid = next_valid;
        }
        if (live && any_endless<16, DTB>(o)) s_special = 1;
        __syncthreads();
        if (__builtin_expect(s_special, 0)) {
            // the tiles again, an element of V's rows at a time: which sums had infinities or NaN
            const int place = hidden(lane), n32 = place & 31, half = place >> 5, row = row0 + wave * 32 + n32;
            const int i = int(fast_div(uint32_t(row < rows ? row : row0), a.div_group));
            const int pos = a.b.positions ? a.b.positions[rq.first + i] : rq.ctx + i;
            Had<16 * DTB> had;
#pragma unroll 1
            for (int t = 0; t < tiles; ++t) {
                if (t % S::kBatch == 0) {
                    __syncthreads();
                    look_up(t / S::kBatch);
                    note_places(t / S::kBatch);
                    note_scales(t / S::kBatch);
                    __syncthreads();
                }
                valid = valid_of(t);
                const uint64_t mine =
                    row < rows ? seen_of(a, rq, r, i, pos, rg.slot(tile_at(t)), valid) >> (4 * half) : 0;
                const int first = (t & (S::kRing - 1)) * KT;
#pragma unroll 1
                for (int t2 = 0; t2 < DTB; ++t2) {
                    const int byte = (32 * t2 + n32) * S::kEl, at = byte < a.c.row_bytes ? byte : 0;
#pragma unroll 1
                    for (int e = 0; e < 2 * ST; ++e) {
                        u32x4 f = {0, 0, 0, 0}, seen;
                        uint32_t some = 0;
#pragma unroll
                        for (int w = 0; w < 4; ++w) {
                            const uint32_t two = uint32_t(mine >> (16 * e + 8 * (w >> 1) + 2 * (w & 1))) & 3u;
                            seen[w] = (two & 1u ? kOne<kBf16> : 0u) | (two & 2u ? kOne<kBf16> << 16 : 0u);
#pragma unroll
                            for (int s = 0; s < 2; ++s) {
                                const int slot = 16 * e + 8 * (w >> 1) + 4 * half + 2 * (w & 1) + s;
                                const char* const from = vb + s_off[first + slot] + at;
                                uint32_t x;
                                if constexpr (k8)
                                    x = times2<kBf16>(widen2<kBf16, kCodes, false>(*reinterpret_cast<const uint8_t*>(from)),
                                                      scale_kind(s_vs[first + slot]), 0.0f) & 0xFFFFu;
                                else
                                    x = *reinterpret_cast<const uint16_t*>(from);
                                f[w] |= (valid >> slot & 1 ? x : 0u) << (16 * s);
                            }
                            some |= nonfinite<kBf16, kCodes16>(f[w]);
                        }
                        if (!__any(some != 0)) continue;
#pragma unroll
                        for (int kind = 1; kind <= 3; ++kind) {
                            f32x16 count;
#pragma unroll
                            for (int i = 0; i < 16; ++i) count[i] = 0.0f;
                            count = mfma32<kBf16>(classify8<kBf16>(f, kind), seen, count);
#pragma unroll
                            for (int i = 0; i < 16; ++i) had.add(16 * t2 + i, count[i], kind);
                        }
                    }
                }
            }
#pragma unroll
            for (int t = 0; t < DTB; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[t][i] = had.of(16 * t + i, o[t][i]);
        }
    }

    l += __shfl_xor(l, 32);
    if constexpr (kLift) l *= 65536.0f;              // 2^kLiftShift
    const float back = kLift ? unlifted(lift) : 1.0f;
    {
        // the row's place, formed anew
        const int place = hidden(lane), half = place >> 5, row = row0 + wave * 32 + (place & 31);
        if (row >= rows) return;
        const int i = int(fast_div(uint32_t(row), a.div_group)), head = h * G + (row - i * G);
        const int64_t token = rq.first + i, at = token * a.q_heads + head;
        if (a.splits > 1) {
            const int64_t pairs = int64_t(a.b.total_tokens) * a.q_heads;
            if (half == 0) {
                a.part_ml[2 * (split * pairs + at)] = reference_of(m, l);
                a.part_ml[2 * (split * pairs + at) + 1] = l;
            }
            if (l == 0.0f) return;
            float* const out = a.part_o + (split * pairs + at) * D;
#pragma unroll
            for (int t = 0; t < DTB; ++t)
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const int d = 32 * t + 8 * b + 4 * half;
                    f32x4 x;
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[i] = kLift ? o[t][4 * b + i] * back : o[t][4 * b + i];
                    if (d < D) *reinterpret_cast<f32x4*>(out + d) = x;
                }
        } else {
            const float inv = l == 0.0f ? 0.0f : back / l;
            uint16_t* const out = a.out + token * a.out_stride + int64_t(head) * D;
#pragma unroll
            for (int t = 0; t < DTB; ++t)
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const int d = 32 * t + 8 * b + 4 * half;
                    const uint2 w = l == 0.0f ? make_uint2(0, 0)
                                              : make_uint2(pack2<kBf16>(o[t][4 * b] * inv, o[t][4 * b + 1] * inv),
                                                           pack2<kBf16>(o[t][4 * b + 2] * inv, o[t][4 * b + 3] * inv));
                    if (d < D) *reinterpret_cast<uint2*>(out + d) = w;
                }
            if (a.lse && half == 0)
                a.lse[at] = l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l) - kShift<kBf16>) * kLn2;
        }
    }
}

template <bool kBf16, int kCodes, int DP, int NW, int kScores>
int go_as(const AttendArgs& a, const AttendPlan& p, void* stream)
{
    const int64_t groups = int64_t(a.c.num_requests) * a.splits * a.c.hd;
    return launch_kernel(kvx_attend_rows_kernel<kBf16, kCodes, DP, NW, kScores>, groups * p.row_tiles, 64 * NW,
                         stream, a, p.row_tiles);
}

template <bool kBf16, int kCodes, int DP, int NW>
int go(const AttendArgs& a, const AttendPlan& p, void* stream)
{
    switch (scores_of(a)) {
    case kWide: return go_as<kBf16, kCodes, DP, NW, kCappedWide>(a, p, stream);
    case kGeneral:
        return a.softcap > 0.0f ? go_as<kBf16, kCodes, DP, NW, kCapped>(a, p, stream)
                                : go_as<kBf16, kCodes, DP, NW, kBiased>(a, p, stream);
    default: return go_as<kBf16, kCodes, DP, NW, kPlain>(a, p, stream);
    }
}

template <bool kBf16, int kCodes>
int pick(const AttendArgs& a, const AttendPlan& p, void* stream)
{
    const bool two = p.tile_rows == 64;
    if (a.c.dim <= 64) return two ? go<kBf16, kCodes, 64, 2>(a, p, stream) : go<kBf16, kCodes, 64, 4>(a, p, stream);
    if (a.c.dim <= 128) return two ? go<kBf16, kCodes, 128, 2>(a, p, stream) : go<kBf16, kCodes, 128, 4>(a, p, stream);
    return two ? go<kBf16, kCodes, 256, 2>(a, p, stream) : go<kBf16, kCodes, 256, 4>(a, p, stream);
}

}  // namespace

template <int kCodes>
int launch_rows(const AttendArgs& a, const AttendPlan& p, int dtype, void* stream)
{
    return dtype == KVX_BF16 ? pick<true, kCodes>(a, p, stream) : pick<false, kCodes>(a, p, stream);
}

}  // namespace kvx
