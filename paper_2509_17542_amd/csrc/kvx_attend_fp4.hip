// Attention of few query rows per KV head over a 4-bit cache: up to 16 rows, the
// tokens of a request times the query heads of a KV head.
//
// Bound by reading K and V once, a quarter of a 16-bit cache's bytes, so what is done
// to a code counts.  A workgroup takes HP KV heads together, whose rows lie side by side
// (whole lines, and one set of statistics for all their rows).  Its 4 waves take tiles of 32
// slots in turn, 128 slots a turn; K and V go from memory to the matrix instructions' registers
// with no stop in LDS, two codes at a time through the conversion that takes their
// group's scale with it:
//   S^T = K Q^T   lane (slot, g) holds 16 bytes of its slot's row, a group; every head's keys meet
//                 all columns, and a lane keeps its own head's sums;
//   O^T = V^T P^T lane (m, g) holds, for the 8 slots whose weights it has, the EL elements
//                 of lane m's place in the HP heads' rows: 16 lanes read them whole.  With 8
//                 columns or fewer each is there twice: pairs of elements go into the product as
//                 they are converted, and the twins' weights take the lower or the upper
//                 one.  More columns take single elements, which v_perm_b32 puts together.  The
//                 result rows belong to the heads of their m; what they hold in columns of
//                 other heads is left.
// The slots' places and scale bytes are looked up 2816 at a time into LDS, the latter while the
// first rows are on their way; a tile's rows are for the whole of the turn before.  Codes are
// finite whatever they are; a value's group that is NaN counts as zero in the products, and
// where there was one a walk over the slots says which rows saw it.
//
// Work is dealt in turns: all requests' turns in a row, cut into as many even ranges as the card
// holds workgroups of a pack of heads at once (a workgroup has a chain of lookups before its
// first turn and a join of its waves after its last: 64 requests of 512..8192 slots in fixed chunks
// of 512 took 97 us, in ranges of 17 turns 77).  A range that holds the end of a request and
// the beginning of the next one is two segments; a segment that is not all of its request leaves
// its sums for kvx_fp4_join_kernel.  Requests of up to 1024 slots have a workgroup each.
//
// Those 64 requests (8 KV heads of 4 query heads, 128 elements, 311 MB) take 73 us and the join
// 5: 4.0 TB/s in all.  With nothing done to the rows once they are there it is 71: what bounds it
// are the loads and, at a range's ends, chains of them (lengths, table, scale bytes, first rows).  A lane
// holds two tiles of rows: 211 registers of 256, fp16 queries 228.  The many-rows kernel takes 183.  One
// request of 120000 slots, fp16, 4 KV heads: 30.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "kvx_attend_dev.h"

namespace kvx {
namespace {

constexpr int kWaves = 4;
constexpr int kWg = 64 * kWaves;
constexpr int kTile = 32;           // slots of a wave's turn
constexpr int kStep = kWaves * kTile;   // of a workgroup's
constexpr int kChunk = 22 * kStep;  // slots whose places and scale bytes are in LDS at once

template <int DP, int HP, bool kDup>
struct Shape {
    static constexpr int kCols = (kDup ? 8 : 16) / HP; // rows of a head, at most
    static constexpr int kLanes = 16 / HP;             // lanes of a head's row of V
    static constexpr int EL = DP / kLanes;             // elements of V in a lane, all of one group
    static constexpr int kSums = kDup ? EL / 2 : EL;   // products of a tile with V
    static constexpr int kVBytes = EL / 2;
    static constexpr int kVWords = (kVBytes + 3) / 4;
    static constexpr int kPieces = DP >= 128 ? DP / 128 : 1;   // of K in a lane, each in one group
    static constexpr int kKWords = DP >= 128 ? 4 : 2;  // of a piece
    static constexpr int kGroups = HP * DP / 32;       // scale bytes of the heads' rows
};

template <int kWords>
struct Row {
    uint32_t w[kWords];
};

// Rows that are read once: non-temporal.
template <int kBytes>
__device__ __forceinline__ Row<(kBytes + 3) / 4> load_row(const char* p)
{
    constexpr int kN = (kBytes + 3) / 4;
    Row<kN> v;
    if constexpr (kBytes == 2) {
        v.w[0] = *reinterpret_cast<const uint16_t*>(p);
    } else if constexpr (kN == 1) {
        v.w[0] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(p));
    } else {
        typedef uint32_t part_t __attribute__((ext_vector_type(kN)));
        const part_t x = __builtin_nontemporal_load(reinterpret_cast<const part_t*>(p));
#pragma unroll
        for (int i = 0; i < kN; ++i) v.w[i] = x[i];
    }
    return v;
}

// In each byte of a word of scale bytes that stand for NaN (above 252), its highest bit.
__device__ __forceinline__ uint32_t no_scales(uint32_t w)
{
    return ((w & 0x7F7F7F7Fu) + 0x03030303u) & w & 0x80808080u;
}

// ---- how work is dealt ----------------------------------------------------------
//
// Turn numbers run through the requests and through each one's slots.  A request has as
// many as its range of slots needs (given positions may narrow a window's: such turns have
// nothing to do) and kSetup more ahead of them, for the lookups and the join that a segment costs
// whatever its length.  Of `total` turns range i of n, n <= total, has [i total / n, (i + 1) total / n);
// each pack of heads has a workgroup to every range, and these read lines that they share (of
// rows shorter than a line, and of scale bytes) at one time and through one L2.
constexpr int kSetup = 3;

__device__ __forceinline__ int turns_of(const AttendArgs& a, int r)
{
    if (r >= a.c.num_requests) return 0;
    const Request rq = request_of(a.c, a.b, r);
    if (rq.n == 0) return 0;
    const int fix = a.prefix ? min(max(a.prefix[r], 0), rq.total) : 0;
    int hi = a.b.tree ? rq.total : min(rq.total, max(rq.ctx + rq.n, fix)), skip = 0;
    if (a.window > 0 && !a.b.positions) {
        const int64_t lo = max(int64_t(0), min(int64_t(rq.ctx) - a.window + 1, int64_t(rq.total)));
        const int pre = (fix + 63) & ~63;
        if (pre < hi) skip = max(0, (int(lo) & ~63) - pre);
        if (pre + skip >= hi) hi = pre, skip = 0;
    }
    return hi > skip ? kSetup + (hi - skip + kStep - 1) / kStep : 0;
}

__device__ __forceinline__ int wave_scan(int x)        // sums of the lanes up to this one
{
    const int lane = int(threadIdx.x) & 63;
    for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(x, o);
        if (lane >= o) x += y;
    }
    return x;
}

// The turns of 64 requests, one to each lane of a wave: its own and those up to it.
struct Turns {
    int mine, upto;
};

__device__ __forceinline__ Turns turns_from(const AttendArgs& a, int r0)
{
    Turns t;
    t.mine = turns_of(a, r0 + (int(threadIdx.x) & 63));
    t.upto = wave_scan(t.mine);
    return t;
}

// Turns of all requests, by a wave; head: those of the first 64.
__device__ __forceinline__ int64_t all_turns(const AttendArgs& a, Turns& head)
{
    head = turns_from(a, 0);
    int64_t sum = __shfl(head.upto, 63);
    for (int r0 = 64; r0 < a.c.num_requests; r0 += 64) sum += __shfl(turns_from(a, r0).upto, 63);
    return sum;
}

struct Unit {
    int r, turns;
    int64_t first;                                     // its first turn
};

// The request that turn `at` belongs to, by a wave; at is below their sum.
__device__ __forceinline__ Unit unit_at(const AttendArgs& a, const Turns& head, int64_t at)
{
    int64_t before = 0;
    Turns t = head;
    for (int r0 = 0; r0 < a.c.num_requests; r0 += 64) {
        if (r0) t = turns_from(a, r0);
        const int64_t end = before + __shfl(t.upto, 63);
        if (at < end) {
            const int l = __builtin_ctzll(__ballot(before + t.upto > at));
            return {r0 + l, __shfl(t.mine, l), before + (__shfl(t.upto, l) - __shfl(t.mine, l))};
        }
        before = end;
    }
    return {0, 0, 0};
}

// The range that has turn `at`.
__device__ __forceinline__ int range_at(int64_t at, int64_t total, int ranges)
{
    return int(((at + 1) * ranges - 1) / total);
}

// Segments of a pack are numbered like its ranges, plus the request's number: no two have the same.
struct Parts {
    float* ml;                                         // [segment][pack][16] pairs
    float* o;                                          // [segment][pack][16][D]
    int2* span;                                        // [request]: first and last range
};

__host__ __device__ inline int64_t parts_count(int64_t ranges, int64_t requests, int packs) { return (ranges + requests) * packs; }

__device__ __forceinline__ Parts parts_of(const AttendArgs& a, int heads)
{
    const int64_t n = parts_count(a.ranges, a.c.num_requests, a.c.hd / heads);
    float* const o = a.part_ml + n * 32;
    return {a.part_ml, o, reinterpret_cast<int2*>(o + n * 16 * a.c.dim)};
}

// ---- the products -----------------------------------------------------------------

template <bool kBf16, int DP, int HP, bool kDup, int kScores, bool kFull>
__global__ void __launch_bounds__(kWg, 2) kvx_attend_fp4_kernel(const AttendArgs a)
{
    using S = Shape<DP, HP, kDup>;
    constexpr int EL = S::EL, kCols = S::kCols, kGroups = S::kGroups, kSums = S::kSums;
    constexpr int kRow = DP + 4;                       // floats of a column's sums: 16 columns in 16 banks
    constexpr bool kTwo = !kBf16;                      // queries in two terms
    constexpr int kScaleBytes = kChunk * kGroups;
    constexpr int kKeyBytes = kChunk * (kScores != kPlain ? 8 : 4) + 2 * kScaleBytes, kSlabBytes = 2 * HP * kCols * kRow * 4;
    __shared__ __attribute__((aligned(16))) char smem[kKeyBytes > kSlabBytes ? kKeyBytes : kSlabBytes];
    __shared__ uint64_t s_valid[kChunk / 64];
    __shared__ float s_ml[kWaves][16][2];
    __shared__ int s_special;
    uint32_t* const s_at = reinterpret_cast<uint32_t*>(smem);   // a slot's row, in groups of 16 bytes
    uint8_t* const s_ks = reinterpret_cast<uint8_t*>(smem + kChunk * 4);
    uint8_t* const s_vs = s_ks + kScaleBytes;
    int32_t* const s_pos = reinterpret_cast<int32_t*>(s_vs + kScaleBytes);

    const int tid = int(threadIdx.x), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n16 = lane & 15, g = lane >> 4;
    const int D = a.c.dim, G = a.group, rg = a.c.row_groups;
    const int packs = a.c.hd / HP;
    const uint8_t* const kgroups = a.c.groups;
    const uint8_t* const vgroups = a.c.groups + a.c.plane_scales * rg;
    const char* const kb = a.c.base;
    const char* const vb = a.c.base + a.c.plane_bytes;

    // neighbours to one XCD
    const uint32_t group = gridDim.x % 8 ? blockIdx.x : blockIdx.x % 8 * (gridDim.x / 8) + blockIdx.x / 8;
    const int range = int(group / uint32_t(packs)), pack = int(group - uint32_t(range) * uint32_t(packs));
    int64_t at = 0, end = 1, total = 0;
    int ranges = 0;
    Turns head = {};
    if (a.ranges) {
        total = all_turns(a, head);
        ranges = int(min(int64_t(a.ranges), total));   // each has a turn at least
        if (range >= ranges) return;
        at = int64_t(range) * total / ranges;
        end = int64_t(range + 1) * total / ranges;
    }
  for (; at < end;) {
    int r = range, turns = INT32_MAX / kStep, t0 = 0, t1 = turns;
    if (a.ranges) {
        const Unit unit = unit_at(a, head, at);
        const int64_t first = unit.first + kSetup;
        r = __builtin_amdgcn_readfirstlane(unit.r);
        turns = __builtin_amdgcn_readfirstlane(unit.turns - kSetup);
        t0 = __builtin_amdgcn_readfirstlane(int(max(at - first, int64_t(0))));
        t1 = __builtin_amdgcn_readfirstlane(int(min(int64_t(turns), end - first)));
        at = min(first + turns, end);
        if (t1 <= t0) continue;                        // nothing but the setup
        if (t0 == 0 && pack == 0 && tid == 0)          // for the join
            parts_of(a, HP).span[r] = make_int2(range, range_at(first + turns - 1, total, ranges));
    } else {
        at = end;
    }
    const int h0 = pack * HP;
    const Request rq = request_of(a.c, a.b, r);
    const int rows = rq.n * G;                         // of a head
    if (rows == 0) return;                             // no turns: a workgroup of its own
    const Range rg_of = range_of(a, rq, r, 0, rq.n - 1);
    const int v0 = t0 * kStep, v1 = min(t1 * kStep, rg_of.len);

    if (tid == 0) s_special = 0;

    // queries: this lane's column, in the element order of K's pieces
    const int col = kDup ? n16 & 7 : n16, twin = kDup ? n16 >> 3 : 0;
    const int col_head = col / kCols, row = col % kCols;
    const bool live = row < rows;
    const int rr = live ? row : 0;
    const int tok = int(fast_div(uint32_t(rr), a.div_group));
    const int head = (h0 + col_head) * G + (rr - tok * G);
    const int qpos = a.b.positions ? a.b.positions[rq.first + tok] : rq.ctx + tok;
    const uint32_t my_half = twin ? 0xFFFF0000u : 0xFFFFu;
    const float slope2 = a.slopes ? a.slopes[head] * kLog2e : 0.0f;
    constexpr int kC = S::kPieces * S::kKWords;        // products of 16 slots with 32 elements
    u32x4 q[kC], q_rest[kTwo ? kC : 1];
    {
        const uint16_t* const src = a.q + int64_t(rq.first + tok) * a.q_stride + int64_t(head) * D;
#pragma unroll
        for (int c = 0; c < kC; ++c) {
            const int d = DP >= 128 ? (c >> 2) * 128 + g * 32 + (c & 3) * 8 : g * 16 + c * 8;
            q[c] = u32x4{0, 0, 0, 0};
            if (live && d < D) q[c] = *reinterpret_cast<const u32x4*>(src + d);
            if constexpr (kTwo)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    uint32_t more;
                    q[c][w] = two_terms(q[c][w], more);
                    q_rest[c][w] = more;
                }
        }
    }
    const ScoreArgs sc = score_args(a);
    f32x4 o[kSums];
    float m = -INFINITY, l = 0.0f;
#pragma unroll
    for (int t = 0; t < kSums; ++t) o[t] = f32x4{0, 0, 0, 0};

    // Loads take no branch: a slot that lies in no page reads the plane's first row and
    // is masked, a lane past a row's end its first piece, which meets q's zeros or is not written.
    constexpr int kKBytes = S::kKWords * 4;
    int k_at[S::kPieces];
#pragma unroll
    for (int p = 0; p < S::kPieces; ++p) {
        k_at[p] = p * 64 + g * kKBytes;
        if (k_at[p] >= a.c.row_bytes) k_at[p] = 0;
    }
    const int my_head = n16 / S::kLanes, my_part = n16 % S::kLanes;
    const bool in_row = my_part * EL < D;
    const int v_at = my_head * a.c.row_bytes + (in_row ? my_part * S::kVBytes : 0);
    const int v_group = my_head * (DP / 32) + (in_row ? my_part * EL / 32 : 0);

    const char* const vb_mine = vb + v_at;
    struct Keys {
        Row<S::kKWords> w[HP][2][S::kPieces];
    };
    struct Values {
        Row<S::kVWords> w[8];
    };
    // A slot's scale bytes of the HP heads; a row's groups lie DP / 32 apart here, whatever D is.
    struct Scales {
        uint32_t w[(kGroups + 3) / 4];
    };
    auto load_scales = [&](const uint8_t* from, Scales& x) {
        if constexpr (kFull) {                         // D is DP: the bytes of the HP heads are whole words
            if constexpr (kGroups == 2) {
                x.w[0] = *reinterpret_cast<const uint16_t*>(from);
            } else {
                typedef uint32_t part_t __attribute__((ext_vector_type(kGroups < 4 ? 1 : kGroups / 4)));
                *reinterpret_cast<part_t*>(x.w) = *reinterpret_cast<const part_t*>(from);
            }
        } else {
#pragma unroll
            for (int i = 0; i < (kGroups + 3) / 4; ++i) x.w[i] = 0;
#pragma unroll
            for (int i = 0; i < kGroups; ++i) {
                const int hh = i / (DP / 32), part = i % (DP / 32);
                if (part < rg) x.w[i >> 2] |= uint32_t(from[hh * rg + part]) << (8 * (i & 3));
            }
        }
    };
    // Places of the slots from c0 on; then, the first rows being on their way, their scale bytes.
    constexpr int kEach = kGroups > 8 ? 2 : 4;         // a thread's slots at once
    auto stage_places = [&](int c0, int c1) {
#pragma unroll 1
        for (int from = c0; from < c1; from += 4 * kWg) {
            int64_t row[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int v = from + k * kWg + tid, j = rg_of.slot(v);
                row[k] = v < c1 && j < rq.total ? slot_row(a.c, r, j) : -1;
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int at = from - c0 + k * kWg + tid;
                if (at >= kChunk) break;               // whole waves
                const uint64_t some = __ballot(row[k] >= 0);
                if (lane == 0) s_valid[at >> 6] = some;
                s_at[at] = row[k] < 0 ? 0u : uint32_t((row[k] + h0) * rg);
                if constexpr (kScores != kPlain) s_pos[at] = place_of(a, rq, rg_of.slot(c0 + at));
            }
        }
    };
    auto stage_scales = [&](int c0, int c1) {
#pragma unroll 1
        for (int first = tid; first < ((c1 - c0 + kTile - 1) & -kTile); first += kEach * kWg) {   // whole tiles
            Scales ks[kEach], vs[kEach];
#pragma unroll
            for (int k = 0; k < kEach; ++k) {
                // 16 bytes of codes have a scale byte
                const uint32_t from = s_at[min(first + k * kWg, kChunk - 1)];
                load_scales(kgroups + from, ks[k]);
                load_scales(vgroups + from, vs[k]);
            }
#pragma unroll
            for (int k = 0; k < kEach; ++k) {
                const int at = first + k * kWg;
                if (at >= kChunk) break;
                // a key's group that is none is NaN in its products, a value's zero
                uint32_t found = 0;
#pragma unroll
                for (int i = 0; i < (kGroups + 3) / 4; ++i) {
                    ks[k].w[i] |= (no_scales(ks[k].w[i]) >> 7) * 0xFFu;
                    const uint32_t none = no_scales(vs[k].w[i]);
                    vs[k].w[i] &= ~((none >> 7) * 0xFFu);
                    found |= none;
                }
                if (found && at < c1 - c0) s_special = 1;
                if constexpr (kGroups >= 4) {
#pragma unroll
                    for (int i = 0; i < kGroups / 4; ++i) {
                        reinterpret_cast<uint32_t*>(s_ks + at * kGroups)[i] = ks[k].w[i];
                        reinterpret_cast<uint32_t*>(s_vs + at * kGroups)[i] = vs[k].w[i];
                    }
                } else {
                    *reinterpret_cast<uint16_t*>(s_ks + at * kGroups) = uint16_t(ks[k].w[0]);
                    *reinterpret_cast<uint16_t*>(s_vs + at * kGroups) = uint16_t(vs[k].w[0]);
                }
            }
        }
    };
    auto load_k = [&](int at, Keys& x) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const char* const from = kb + (uint64_t(s_at[at + 16 * e + n16]) << 4);
#pragma unroll
            for (int hh = 0; hh < HP; ++hh)
#pragma unroll
                for (int p = 0; p < S::kPieces; ++p)
                    x.w[hh][e][p] = load_row<kKBytes>(from + hh * a.c.row_bytes + k_at[p]);
        }
    };
    auto load_v = [&](int at, Values& x) {             // slots 4 g .. 4 g + 3 of each half
#pragma unroll
        for (int j = 0; j < 8; ++j)
            x.w[j] = load_row<S::kVBytes>(vb_mine + (uint64_t(s_at[at + 16 * (j >> 2) + 4 * g + (j & 3)]) << 4));
    };

    // The tile at v, place `at` of the chunk.
    auto turn = [&](int v, int at, const Keys& x, const Values& y) {
        const uint32_t valid = uint32_t(__builtin_amdgcn_readfirstlane(int(uint32_t(s_valid[at >> 6] >> (at & 32)))));
        const int j0 = rg_of.slot(v);
        const bool whole = j0 >= rg_of.all_lo && j0 + kTile <= rg_of.all_hi && valid == ~0u;
        float s[2][4];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const uint8_t* const scale = s_ks + (at + 16 * e + n16) * kGroups;
#pragma unroll
            for (int hh = 0; hh < HP; ++hh) {
                f32x4 acc = {0, 0, 0, 0};
#pragma unroll
                for (int p = 0; p < S::kPieces; ++p) {
                    const int group = hh * (DP / 32) + (DP >= 128 ? 4 * p + g : g >> 1);
                    const float by = __uint_as_float(uint32_t(scale[group]) << 23);
#pragma unroll
                    for (int c = 0; c < S::kKWords; ++c) {
                        const u32x4 f = widen4x8(x.w[hh][e][p].w[c], by);
                        acc = mfma16<true>(f, q[p * S::kKWords + c], acc);
                        if constexpr (kTwo) acc = mfma16<true>(f, q_rest[p * S::kKWords + c], acc);
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) s[e][i] = hh == 0 || col_head == hh ? acc[i] : s[e][i];
            }
        }
        float top = -INFINITY;
        uint32_t mine = ~0u;
        if (!whole) mine = live ? uint32_t(seen_of(a, rq, r, tok, qpos, j0, valid)) >> (4 * g) : 0u;
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (kScores == kPlain)
                    s[e][i] *= sc.c2;
                else
                    s[e][i] = general_score<kScores>(sc, s[e][i], slope2, qpos - s_pos[at + 16 * e + 4 * g + i]);
                if (!whole && !(mine >> (16 * e + i) & 1u)) s[e][i] = -INFINITY;
                top = fmaxf(top, s[e][i]);
            }
        if (__any(top > m + kSlack)) {
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float to = fmaxf(m, top);
            const float alpha = to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - to);
            l *= alpha;
            m = to;
#pragma unroll
            for (int t = 0; t < kSums; ++t) o[t] *= alpha;
        }
        const float base = m == -INFINITY ? 0.0f : m;
        // Weights in two terms.  Twin columns take a pair of V's elements, the first its lower one,
        // the other its upper: then a pair goes into the product as it is converted.
        constexpr int kWords = kDup ? 8 : 4;
        uint32_t pf[kWords], rest[kWords];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            float p[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                p[i] = __builtin_amdgcn_exp2f(s[w >> 1][2 * (w & 1) + i] - base);
                l += p[i];
                if constexpr (kDup) {
                    const uint32_t both = pack2<true>(p[i], p[i]);
                    const float more = p[i] - value16<true>(both >> 16);
                    pf[2 * w + i] = both & my_half;
                    rest[2 * w + i] = pack2<true>(more, more) & my_half;
                }
            }
            if constexpr (!kDup) {
                pf[w] = pack2<true>(p[0], p[1]);
                rest[w] = pack2<true>(p[0] - value16<true>(pf[w] & 0xFFFFu), p[1] - value16<true>(pf[w] >> 16));
            }
        }
        float by[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            by[j] = __uint_as_float(uint32_t(s_vs[(at + 16 * (j >> 2) + 4 * g + (j & 3)) * kGroups + v_group]) << 23);
        // two elements at a time: a byte of codes of each of the 8 slots
#pragma unroll
        for (int t = 0; t < EL; t += 2) {
            uint32_t two[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t w = y.w[j].w[t >> 3];
                two[j] = (t & 6) == 0 ? widen4<0>(w, by[j]) : (t & 6) == 2 ? widen4<1>(w, by[j])
                         : (t & 6) == 4 ? widen4<2>(w, by[j]) : widen4<3>(w, by[j]);
            }
            if constexpr (kDup) {
#pragma unroll
                for (int k = 0; k < 8; k += 4) {
                    const u32x4 f = {two[k], two[k + 1], two[k + 2], two[k + 3]};
                    o[t / 2] = mfma16<true>(f, u32x4{pf[k], pf[k + 1], pf[k + 2], pf[k + 3]}, o[t / 2]);
                    o[t / 2] = mfma16<true>(f, u32x4{rest[k], rest[k + 1], rest[k + 2], rest[k + 3]}, o[t / 2]);
                }
            } else {
                u32x4 f0, f1;
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    f0[p] = pair16<false>(two[2 * p], two[2 * p + 1]);
                    f1[p] = pair16<true>(two[2 * p], two[2 * p + 1]);
                }
                const u32x4 a0 = {pf[0], pf[1], pf[2], pf[3]}, a1 = {rest[0], rest[1], rest[2], rest[3]};
                o[t] = mfma16<true>(f0, a0, o[t]);
                o[t + 1] = mfma16<true>(f1, a0, o[t + 1]);
                o[t] = mfma16<true>(f0, a1, o[t]);
                o[t + 1] = mfma16<true>(f1, a1, o[t + 1]);
            }
        }
    };

    for (int c0 = v0; c0 < v1; c0 += kChunk) {
        const int c1 = min(c0 + kChunk, v1);
        __syncthreads();                               // the last ones' places are read
        stage_places(c0, c1);
        __syncthreads();
        // a tile's rows are on their way for the whole of the turn before
        int v = c0 + wave * kTile;
        Keys x;
        Values y;
        const int start = v < c1 ? v - c0 : 0;
        load_k(start, x);
        load_v(start, y);
        stage_scales(c0, c1);
        __syncthreads();
#pragma unroll 1
        for (; v < c1; v += kStep) {
            const int next = v + kStep < c1 ? v + kStep : v;
            Keys x1;
            Values y1;
            load_k(next - c0, x1);
            load_v(next - c0, y1);
            turn(v, v - c0, x, y);
            x = x1;
            y = y1;
        }
    }
    // which groups of values that this column saw are NaN
    uint32_t nan = 0;
    __syncthreads();
    if (__builtin_expect(s_special, 0)) {
        for (int v = v0 + wave * kTile; v < v1; v += kStep) {
            const int j = rg_of.slot(v + (lane & 31));
            const int64_t row = v + (lane & 31) < v1 && j < rq.total ? slot_row(a.c, r, j) : -1;
            const uint32_t there = uint32_t(__ballot(row >= 0));
            Scales z;
            load_scales(vgroups + (row < 0 ? 0 : row + h0) * rg, z);
            uint32_t marks = 0;
#pragma unroll
            for (int i = 0; i < kGroups; ++i) marks |= ((z.w[i >> 2] >> (8 * (i & 3)) & 255u) > 252u ? 1u : 0u) << i;
            const uint32_t mine = live ? uint32_t(seen_of(a, rq, r, tok, qpos, rg_of.slot(v), there)) : 0u;
            for (int k = 0; k < kTile; ++k) {
                const uint32_t of = uint32_t(__shfl(int(marks), k));
                if (mine >> k & 1u) nan |= of;
            }
        }
    }

    // the waves' sums, joined through LDS two at a time
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    m = reference_of(m, l);
    if (g == 0) {
        s_ml[wave][n16][0] = m;
        s_ml[wave][n16][1] = l;
    }
    __syncthreads();
    float* const slab = reinterpret_cast<float*>(smem) + (wave & 1) * HP * kCols * kRow;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, s_ml[w][n16][0]);
    const float scale = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - top);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        if ((wave >> 1) == half) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int place = 4 * g + i;           // result row: lane m of V
                if (place / S::kLanes == col_head) {
                    const int part = place % S::kLanes;
                    const bool none = nan >> (col_head * (DP / 32) + part * EL / 32) & 1u;
                    float* const to = slab + col * kRow + part * EL + twin;
#pragma unroll
                    for (int t = 0; t < kSums; ++t) {
                        const float x = none ? NAN : o[t][i] * scale;
                        float& at = to[kDup ? 2 * t : t];
                        at = half == 0 ? x : at + x;
                    }
                }
            }
        }
        __syncthreads();
    }
    const float* const sum = reinterpret_cast<const float*>(smem);
    for (int i = tid; i < HP * kCols * (DP / 8); i += kWg) {
        const int col = i / (DP / 8), d = i % (DP / 8) * 8, hh = col / kCols, mine = col % kCols;
        if (mine >= rows || d >= D) continue;
        float most = -INFINITY, total_l = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) most = fmaxf(most, s_ml[w][col][0]);
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
            total_l += s_ml[w][col][0] == -INFINITY ? 0.0f : s_ml[w][col][1] * __builtin_amdgcn_exp2f(s_ml[w][col][0] - most);
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = sum[col * kRow + d + e] + sum[(HP * kCols + col) * kRow + d + e];
        if (t0 > 0 || t1 < turns) {
            const Parts parts = parts_of(a, HP);
            const int64_t part = ((int64_t(range) + r) * packs + pack) * 16 + col;
            float4* const out = reinterpret_cast<float4*>(parts.o + part * D + d);
            out[0] = make_float4(x[0], x[1], x[2], x[3]);
            out[1] = make_float4(x[4], x[5], x[6], x[7]);
            if (d == 0) {
                parts.ml[2 * part] = reference_of(most, total_l);
                parts.ml[2 * part + 1] = total_l;
            }
        } else {
            const int t = int(fast_div(uint32_t(mine), a.div_group));
            const int64_t token = rq.first + t, qh = (h0 + hh) * G + (mine - t * G);
            const float inv = total_l == 0.0f ? 0.0f : 1.0f / total_l;
            u32x4 w;
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = total_l == 0.0f ? 0u : pack2<kBf16>(x[2 * e] * inv, x[2 * e + 1] * inv);
            *reinterpret_cast<u32x4*>(a.out + token * a.out_stride + qh * D + d) = w;
            if (a.lse && d == 0)
                a.lse[token * a.q_heads + qh] = total_l == 0.0f ? -INFINITY : (most + __builtin_amdgcn_logf(total_l)) * kLn2;
        }
    }
    __syncthreads();                                   // the sums are read: the next segment's places go there
  }
}

// ---- segments joined ------------------------------------------------------------
//
// As kvx_join_kernel does: a wave (many segments: a workgroup's four) per token and query head; its
// segments' sums are brought to the largest reference and added in a fixed order.  A
// request that sees no slot at all has no turn: its results are written here.
template <bool kBf16, int kJoin>
__global__ void __launch_bounds__(kWg) kvx_fp4_join_kernel(const AttendArgs a, int heads, int cols, int lg_lanes)
{
    __shared__ __attribute__((aligned(16))) float s_acc[kWaves][256];
    __shared__ float s_top[kWaves], s_sum[kWaves];
    const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) >> 6;
    const int64_t unit = kJoin == 4 ? int64_t(blockIdx.x) : int64_t(blockIdx.x) * kWaves + wave;
    const int part = kJoin == 4 ? wave : 0;
    const int64_t row = unit / a.q_heads;
    const int r = int(row / a.b.max_tokens), tok = int(row - int64_t(r) * a.b.max_tokens);
    if (r >= a.c.num_requests) return;
    const Request rq = request_of(a.c, a.b, r);
    const int head = int(unit - row * a.q_heads), D = a.c.dim, G = a.group, packs = a.c.hd / heads;
    const int kv = head / G, pack = kv / heads;
    const Parts parts = parts_of(a, heads);
    const int2 span = parts.span[r];             // of a request without turns: anything
    if (tok >= rq.n) return;
    const int64_t token = rq.first + tok, at = token * a.q_heads + head;
    uint16_t* const out = a.out + token * a.out_stride + int64_t(head) * D;
    if (turns_of(a, r) == 0) {
        for (int d = lane; d < D; d += 64) out[d] = 0;
        if (a.lse && lane == 0) a.lse[at] = -INFINITY;
        return;
    }
    const int w0 = span.x, w1 = span.y;
    if (w0 == w1) return;                              // written already
    // segment of range w: its column's place
    const int64_t wide = int64_t(packs) * 16;
    const int64_t place = (int64_t(r) * packs + pack) * 16 + (kv - pack * heads) * cols + tok * G + (head - kv * G);
    const float2* const ml = reinterpret_cast<const float2*>(parts.ml) + place;
    // this wave's segments: [begin, end)
    const int n = w1 - w0 + 1, begin = w0 + n * part / kJoin, end = w0 + n * (part + 1) / kJoin;
    float top = -INFINITY;
    for (int w = begin + lane; w < end; w += 64) top = fmaxf(top, ml[w * wide].x);
    for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    if constexpr (kJoin == 4) {
        if (lane == 0) s_top[wave] = top;
        __syncthreads();
        top = fmaxf(fmaxf(s_top[0], s_top[1]), fmaxf(s_top[2], s_top[3]));
    }
    const int lanes = 1 << lg_lanes, d = 4 * (lane & (lanes - 1)), step = 64 >> lg_lanes;
    float acc[4] = {}, sum = 0.0f;
    for (int base = begin; base < end; base += 64) {
        const float2 v = base + lane < end ? ml[(base + lane) * wide] : make_float2(-INFINITY, 0.0f);
        // a segment that saw nothing left no sum: -1
        const float f = v.x == -INFINITY ? -1.0f : __builtin_amdgcn_exp2f(v.x - top);
        sum += f < 0.0f ? 0.0f : v.y * f;
        const int many = min(64, end - base);
        // rows in flight: 30.2 us for one request of 120000 slots, 31.0 with 4
        constexpr int kFlight = kJoin == 4 ? 16 : 4;
        for (int s = 0; s < many; s += kFlight * step) {
            float4 x[kFlight];
            float w[kFlight];
#pragma unroll
            for (int k = 0; k < kFlight; ++k) {
                const int mine = s + k * step + (lane >> lg_lanes);
                const float weight = __shfl(f, mine & 63);
                w[k] = mine < many ? weight : -1.0f;
                x[k] = *reinterpret_cast<const float4*>(
                    parts.o + ((base + min(mine, many - 1)) * wide + place) * D + (d < D ? d : 0));
            }
#pragma unroll
            for (int k = 0; k < kFlight; ++k)
                if (!(w[k] < 0.0f))
                    acc[0] += weighted(x[k].x, w[k]), acc[1] += weighted(x[k].y, w[k]),
                        acc[2] += weighted(x[k].z, w[k]), acc[3] += weighted(x[k].w, w[k]);
        }
    }
    for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
    for (int o = lanes; o < 64; o <<= 1)
#pragma unroll
        for (int k = 0; k < 4; ++k) acc[k] += __shfl_xor(acc[k], o);
    if constexpr (kJoin == 4) {
        if (lane == 0) s_sum[wave] = sum;
        if (lane < lanes) *reinterpret_cast<float4*>(&s_acc[wave][d]) = make_float4(acc[0], acc[1], acc[2], acc[3]);
        __syncthreads();
        if (wave != 0) return;
        sum = (s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            acc[k] = lane < lanes ? (s_acc[0][d + k] + s_acc[1][d + k]) + (s_acc[2][d + k] + s_acc[3][d + k]) : 0.0f;
    }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    if (lane < lanes && d < D)
        *reinterpret_cast<uint2*>(out + d) = sum == 0.0f ? make_uint2(0, 0)
                                                         : make_uint2(pack2<kBf16>(acc[0] * inv, acc[1] * inv),
                                                                      pack2<kBf16>(acc[2] * inv, acc[3] * inv));
    if (a.lse && lane == 0) a.lse[at] = sum == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

template <bool kBf16, int DP, int HP, bool kDup, int kScores>
int go_as(const AttendArgs& a, void* stream)
{
    const int64_t grid = (a.ranges ? a.ranges : int64_t(a.c.num_requests)) * (a.c.hd / HP);
    return a.c.dim == DP ? launch_kernel(kvx_attend_fp4_kernel<kBf16, DP, HP, kDup, kScores, true>, grid, kWg, stream, a)
                         : launch_kernel(kvx_attend_fp4_kernel<kBf16, DP, HP, kDup, kScores, false>, grid, kWg, stream, a);
}

template <bool kBf16, int DP, int HP, bool kDup>
int go(const AttendArgs& a, void* stream)
{
    switch (scores_of(a)) {
    case kWide: return go_as<kBf16, DP, HP, kDup, kWide>(a, stream);
    case kGeneral: return go_as<kBf16, DP, HP, kDup, kGeneral>(a, stream);
    default: return go_as<kBf16, DP, HP, kDup, kPlain>(a, stream);
    }
}

template <bool kBf16>
int pick(const AttendArgs& a, const AttendPlan& p, void* stream)
{
    if (p.rows * p.heads > 8)
        return a.c.dim > 128 ? go<kBf16, 256, 1, false>(a, stream)
               : a.c.dim > 64 ? go<kBf16, 128, 1, false>(a, stream) : go<kBf16, 64, 1, false>(a, stream);
    if (a.c.dim > 128) return go<kBf16, 256, 1, true>(a, stream);
    if (a.c.dim > 64) return p.heads == 2 ? go<kBf16, 128, 2, true>(a, stream) : go<kBf16, 128, 1, true>(a, stream);
    return p.heads == 4 ? go<kBf16, 64, 4, true>(a, stream)
           : p.heads == 2 ? go<kBf16, 64, 2, true>(a, stream) : go<kBf16, 64, 1, true>(a, stream);
}

// by the segments of a request, about
bool join_by_four(int64_t ranges, int64_t requests) { return ranges > 16 * requests; }

template <bool kBf16>
int join(const AttendArgs& a, const AttendPlan& p, void* stream)
{
    int lg_lanes = 0;
    while ((4 << lg_lanes) < a.c.dim) ++lg_lanes;
    const int cols = (p.rows * p.heads > 8 ? 16 : 8) / p.heads;
    const int64_t units = int64_t(a.c.num_requests) * a.b.max_tokens * a.q_heads;
    if (join_by_four(p.ranges, a.c.num_requests))
        return launch_kernel(kvx_fp4_join_kernel<kBf16, 4>, units, kWg, stream, a, p.heads, cols, lg_lanes);
    return launch_kernel(kvx_fp4_join_kernel<kBf16, 1>, (units + kWaves - 1) / kWaves, kWg, stream, a, p.heads, cols, lg_lanes);
}

}  // namespace

void plan_few_fp4(const kvx_cache& c, const kvx_batch& b, AttendPlan& p)
{
    // Heads of a workgroup: as many as leave every column its twin, up to 256 elements.
    p.heads = c.head_dim > 128 ? 1 : c.head_dim > 64 ? 2 : 4;
    while (p.heads > 1 && (c.num_kv_heads % p.heads || p.rows * p.heads > 8)) p.heads >>= 1;
    // A workgroup to each request's pack: short ones, and so many that the card evens them out and
    // finding a range's place among them would cost (8 KV heads of 4 query heads, 128 elements: 512 requests of
    // 1100..1300 slots 159 us, 193 in ranges, of 500..4000 294 and 308; 256 of 500..4000 174 and 164).  Where
    // one of so many is far longer than the others it is what a call takes: 60000 slots among 511 requests of
    // 1000 808 us, 184 in ranges; the host does not know lengths.  Fewer heads to each where they do not fill the card.
    const int64_t requests = c.num_requests, turns = (int64_t(b.max_context) + kStep - 1) / kStep;
    const bool single = turns <= 8 || requests >= 512 || requests * (c.num_kv_heads / p.heads) >= 1024;
    while (single && p.heads > 1 && requests * (c.num_kv_heads / p.heads) < 256) p.heads >>= 1;
    // two workgroups to a CU
    p.ranges = single ? 0 : int(std::max<int64_t>(1, std::min<int64_t>(512 / (c.num_kv_heads / p.heads), requests * turns / 2)));
}

uint64_t workspace_fp4(const kvx_cache& c, const AttendPlan& p)
{
    if (p.ranges == 0) return 0;
    return uint64_t(parts_count(p.ranges, c.num_requests, c.num_kv_heads / p.heads)) * 16 * (2 + uint64_t(c.head_dim)) * 4 +
           uint64_t(c.num_requests) * 8;
}

double threads_fp4(const kvx_cache& c, const kvx_batch& b, int32_t q_heads, const AttendPlan& p)
{
    const double packs = c.num_kv_heads / p.heads;
    if (p.ranges == 0) return c.num_requests * packs * kWg;
    const double units = double(c.num_requests) * b.max_tokens * q_heads;
    return std::max(p.ranges * packs * kWg, join_by_four(p.ranges, c.num_requests) ? units * kWg : units * 64 + kWg);
}

int launch_few_fp4(const AttendArgs& a, const AttendPlan& p, int dtype, void* stream)
{
    const bool bf = dtype == KVX_BF16;
    const int err = bf ? pick<true>(a, p, stream) : pick<false>(a, p, stream);
    if (err || p.ranges == 0) return err;
    return bf ? join<true>(a, p, stream) : join<false>(a, p, stream);
}

}  // namespace kvx
