// kvx_verify: drafted tokens against the target's logits.
//
// A row's softmax needs one pass over its logits, and that is what bounds a call:
//   parts     every row is cut into parts of 4096 logits; a wave takes one, finds its
//             largest, and sums exp((l - top) / T) with all of the part in registers;
//   siblings  (draft's logits given, trees) sum of max(r - q, 0) for every refusal that
//             another child may follow;
//   walk      a workgroup per request joins its rows' parts, decides for every token
//             whether its parent would accept it (that does not depend on the path), and
//             follows the path from the first; without a draft it draws the next token too:
//             the part by the parts' sums, the token by a scan over that part;
//   residual  (draft's logits given) the sums of max(r - q, 0) after the last token;
//   draw      (draft's logits given) the next token by those.
// The next token is the place where a sum over up to V terms passes a given share of
// the whole: an error of 1e-7 of it, as of fp32 exponentials, moves thousands of such
// borders by that much, so all sums are of 64 bits, from exponentials of 2e-13, and a
// request has the same answer in a call of any size.  80 million logits of bf16 take 67 us, 2.4
// TB/s (41 with fp32 exponentials, summed eight at a time in fp32).
// 64 chains of 2..9 tokens over 128256 logits with a draft's take 110 us, four tokens over 32000
// logits 21, nearly all of it launches and chains of lookups.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "kvx_ops_dev.h"
#include "kvx_verify_internal.h"

namespace kvx {
namespace {

constexpr int kWaves = 4;
constexpr int kWg = 64 * kWaves;
constexpr int kWalk = 512;               // threads of a request's workgroup

enum Logits : int { kF16 = 0, kB16 = 1, kF32 = 2 };

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <int kType>
constexpr int kSize = kType == kF32 ? 4 : 2;
template <int kType>
constexpr int kVec = 16 / kSize<kType>;  // logits of 16 bytes

template <int kType>
__device__ __forceinline__ float logit(const char* row, int v)
{
    if constexpr (kType == kF32) return reinterpret_cast<const float*>(row)[v];
    return value16<kType == kB16>(reinterpret_cast<const uint16_t*>(row)[v]);
}

// element e of 16 bytes
template <int kType>
__device__ __forceinline__ float element(const u32x4& w, int e)
{
    if constexpr (kType == kF32) return __uint_as_float(w[e]);
    return value16<kType == kB16>((w[e >> 1] >> (16 * (e & 1))) & 0xFFFFu);
}

// 16 bytes of a row, which need not be aligned to more than an element
__device__ __forceinline__ u32x4 load16(const char* p)
{
    u32x4 w;
    __builtin_memcpy(&w, p, 16);
    return w;
}

// exp2(x / 256) to 1.5e-13, -2.6e5 <= x <= 256; x = 256 n + j + f, |f| <= 1/2: 2^(j / 256) out of
// a table, the series of exp(f ln 2 / 256), whose first term left out is (ln 2 / 512)^4 / 24, and
// n added to the exponent.  Adding 1.5 x 2^52 rounds x to an integer, which lies in the low word.
constexpr int kTable = 256;
constexpr double kLeast = -2.5e5;

__device__ __forceinline__ double exp2_near(const double* table, double x)
{
    constexpr double u = 0.69314718055994530942 / kTable;
    const double whole = x + 0x1.8p52, f = x - (whole - 0x1.8p52);
    const int i = int(uint32_t(__builtin_bit_cast(uint64_t, whole)));
    double y = __builtin_fma(f, u * u * u / 6, u * u / 2);
    y = __builtin_fma(f, y, u);
    y = __builtin_fma(f, y, 1.0);
    const uint64_t w = __builtin_bit_cast(uint64_t, table[i & (kTable - 1)] * y);
    return __builtin_bit_cast(double, uint64_t(uint32_t(w >> 32) + (uint32_t(i & -kTable) << 12)) << 32 | uint32_t(w));
}

// The same for any x <= 256, 0 below 2^-976.
__device__ __forceinline__ double exp2_256th(const double* table, double x)
{
    const double y = exp2_near(table, fmax(x, kLeast));
    return x < kLeast ? 0.0 : y;
}

__device__ __forceinline__ void fill_table(double* table)
{
    for (int i = int(threadIdx.x); i < kTable; i += int(blockDim.x)) table[i] = exp2(double(i) / kTable);
}

// 256 log2(e) / T.  0: greedy
__device__ __forceinline__ double rate_of(const VerifyArgs& a, int r)
{
    const float t = a.temperatures ? a.temperatures[r] : 1.0f;
    if (!(t >= 0x1p-60f)) return 0.0;
    return 369.32993046757462751 / double(fminf(t, 0x1p60f));
}

struct Drafts {
    int first, n;
};

__device__ __forceinline__ Drafts drafts_of(const VerifyArgs& a, int r)
{
    const int s0 = min(max(a.starts[r], 0), a.total_tokens);
    const int s1 = min(max(a.starts[r + 1], s0), a.total_tokens);
    return {s0, min(s1 - s0, a.max_tokens)};
}

// the token that token i of a request follows, or -1
__device__ __forceinline__ int parent_of(const VerifyArgs& a, int first, int i)
{
    if (i == 0) return -1;
    if (!a.parents) return i - 1;
    const int p = a.parents[first + i];
    return p >= 0 && p < i ? p : -1;
}

__device__ __forceinline__ double wave_sum(double x)
{
    for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
    return x;
}

__device__ __forceinline__ const char* row_of(const VerifyArgs& a, int side, int64_t row, int size)
{
    return side ? a.draft + row * a.draft_stride * size : a.logits + row * a.stride * size;
}

// ---- parts ---------------------------------------------------------------------

constexpr int kLeaf = 1 << 30;           // VerifyArgs::last: nothing was refused there

template <int kType>
__global__ void __launch_bounds__(kWg, 4) kvx_verify_parts_kernel(const VerifyArgs a)
{
    constexpr int kV = kVec<kType>, kEach = kPart / 64 / kV;
    __shared__ double s_table[kTable];
    fill_table(s_table);
    __syncthreads();
    const int lane = int(threadIdx.x) & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
    const int64_t unit = int64_t(blockIdx.x) * kWaves + wave, rows = unit / a.parts;
    const int c = int(unit - rows * a.parts), side = rows >= a.total_tokens;
    const int64_t index = rows - (side ? a.total_tokens : 0);
    if (index >= a.total_tokens || (side && !a.draft)) return;
    const int row = int(index), r = request_at(a.starts, a.num_requests, row);
    if (r < 0 || r >= a.num_requests) return;
    const Drafts d = drafts_of(a, r);
    const int at = row - d.first;
    if (at >= d.n) return;
    const double rate = rate_of(a, r);
    if (side) {
        // a draft's row counts where it has children
        bool some = false;
        if (rate != 0.0) {
            if (!a.parents)
                some = at + 1 < d.n;
            else
                for (int i = at + 1; i < d.n && !some; i += 64)
                    some = __any(i + lane < d.n && parent_of(a, d.first, i + lane) == at) != 0;
        }
        if (!some) return;
    }
    const char* const x = row_of(a, side, row, kSize<kType>) + int64_t(c) * kPart * kSize<kType>;
    const int n = min(kPart, a.vocab - c * kPart);
    u32x4 w[kEach];
    if (n == kPart) {
#pragma unroll
        for (int k = 0; k < kEach; ++k) w[k] = load16(x + (k * 64 + lane) * 16);
    } else {
        // The last 16 bytes of the row again where it ends, their elements that others have, and
        // what lies past the end, -infinity.
        constexpr uint32_t none = kType == kF32 ? 0xFF800000u : kType == kB16 ? 0xFF80u : 0xFC00u;
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            const int v = (k * 64 + lane) * kV, from = max(min(v, n - kV), 0);
            if (n >= kV) {
                w[k] = load16(x + from * kSize<kType>);
            } else {
                w[k] = u32x4{0, 0, 0, 0};
                for (int e = 0; e < n; ++e) {
                    const uint32_t h = kType == kF32 ? reinterpret_cast<const uint32_t*>(x)[e]
                                                     : reinterpret_cast<const uint16_t*>(x)[e];
                    const int word = kType == kF32 ? e : e >> 1;
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[k][i] |= i == word ? h << (kType == kF32 ? 0 : 16 * (e & 1)) : 0u;
                }
            }
            // elements [least, most) of these are this lane's
            const int least = v - from, most = n - from;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (kType == kF32) {
                    if (i < least || i >= most) w[k][i] = none;
                } else {
                    if (2 * i < least || 2 * i >= most) w[k][i] = (w[k][i] & 0xFFFF0000u) | none;
                    if (2 * i + 1 < least || 2 * i + 1 >= most) w[k][i] = (w[k][i] & 0xFFFFu) | none << 16;
                }
            }
        }
    }
    // the largest; NaN where one is NaN
    float top = -INFINITY;
#pragma unroll
    for (int k = 0; k < kEach; ++k)
#pragma unroll
        for (int e = 0; e < kV; ++e) top = __builtin_elementwise_maximum(top, element<kType>(w[k], e));
    for (int o = 32; o; o >>= 1) top = __builtin_elementwise_maximum(top, __shfl_xor(top, o));
    const bool bad = !(top < INFINITY);
    int first = INT32_MAX;
    if (rate == 0.0) {
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            const int from = max(min((k * 64 + lane) * kV, n - kV), 0);   // where its 16 bytes lie
#pragma unroll
            for (int e = 0; e < kV; ++e)
                if (element<kType>(w[k], e) == top) first = min(first, c * kPart + from + e);
        }
        for (int o = 32; o; o >>= 1) first = min(first, __shfl_xor(first, o));
    }
    double sum = 0.0;
    if (bad || top == -INFINITY) {
        sum = 0.0;
    } else if (rate == 0.0) {
        sum = lane == 0 ? 1.0 : 0.0;
    } else {
        // What is far below weighs 2^-976 here.  The difference is formed first: a multiply-add of the
        // product and top's would save an instruction, but takes a rate cut to 40 bits, 1e-12 of the
        // distance from the top.
#pragma unroll
        for (int k = 0; k < kEach; ++k)
#pragma unroll
            for (int e = 0; e < kV; ++e) {
                const double x = (double(element<kType>(w[k], e)) - double(top)) * rate;
                sum += exp2_near(s_table, fmax(x, kLeast));
            }
    }
    sum = wave_sum(sum);
    if (bad) sum = NAN;
    if (lane == 0) a.part[side][int64_t(row) * a.parts + c] = Part{sum, top, first};
}

// ---- what a row is ---------------------------------------------------------------

// A row's softmax: weight exp2((l - top) rate / 256) of sum `sum`; sum 0: no distribution.
struct Whole {
    double sum;
    float top;
    int32_t at;                          // greedy: the first of the largest
};

// Joins a row's parts; by `lanes` (a power of two, 64 at most) lanes of a wave, all of which get it.
__device__ __forceinline__ Whole join(const Part* part, int parts, double rate, const double* table, int lane, int lanes)
{
    float top = -INFINITY;
    for (int c = lane; c < parts; c += lanes) top = fmaxf(top, part[c].top);
    for (int o = lanes >> 1; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    double sum = 0.0;
    int at = INT32_MAX;
    for (int c = lane; c < parts; c += lanes) {
        const Part p = part[c];
        const double by = exp2_256th(table, p.top == -INFINITY ? 2 * kLeast : (double(p.top) - double(top)) * rate);
        sum += p.sum * (p.top == -INFINITY ? 1.0 : by);
        if (p.top == top) at = min(at, p.at);
    }
    for (int o = lanes >> 1; o; o >>= 1) {
        sum += __shfl_xor(sum, o);
        at = min(at, __shfl_xor(at, o));
    }
    if (!(sum > 0.0) || !(sum < INFINITY) || !(__builtin_fabsf(top) < INFINITY)) sum = 0.0;
    return {sum, top, at};
}

// a logit's share of its row
__device__ __forceinline__ double share(float l, float top, double rate, double by, const double* table)
{
    return exp2_256th(table, (double(l) - double(top)) * rate) * by;
}

// What refusing children leaves of r.  Child j's refusal makes r(v) left(j) max(r(v) - q(v) by(j), 0), the
// factor `left` bringing its sum to 1, from r = p on.  All of them come to one term:
//   r(v) = A max(p(v) - q(v) B, 0),   A = left(0) .. left(j),
//   B = by(0) + by(1) / left(0) + .. + by(j) / (left(0) .. left(j - 1)),
// since max(A max(x, 0) - y, 0) = A max(x - y / A, 0) for positive A and y.  Siblings drawn without
// replacement take their tokens out of q: of child i's token B ends with by(i).  So a refusal's pass over
// a row takes the same work whatever the number of children (a token's children times V in all;
// replaying the refusals before each took 59 ms for 128 children and 32000 logits, 1.6 so).
__device__ __forceinline__ double rest(double p, double q, double upto)
{
    return fmax(__builtin_fma(-upto, q, p), 0.0);
}

// The children of a token, in LDS: their numbers, tokens, and the factors above.
struct Children {
    int number[kMaxDrafted];
    int token[kMaxDrafted];
    double by[kMaxDrafted];              // what q is multiplied by at that child; then the B above up to it
    double left[kMaxDrafted];
    uint8_t dull[kMaxDrafted];           // a token that an earlier sibling is, or none of the vocabulary
    int count;
};

// The children of token `at` in ascending order, by a workgroup of whole waves (all threads call).
__device__ __forceinline__ void list_children(const VerifyArgs& a, const Drafts& d, int at, Children& s)
{
    __syncthreads();
    if (threadIdx.x < 64) {
        const int lane = int(threadIdx.x);
        int count = 0;
        const int end = a.parents ? d.n : min(d.n, at + 2);
        for (int i0 = at + 1; i0 < end; i0 += 64) {
            const int i = i0 + lane;
            const bool mine = i < end && parent_of(a, d.first, i) == at;
            const uint64_t m = __ballot(mine);
            if (mine) {
                const int k = count + __popcll(m & ((uint64_t(1) << lane) - 1));
                s.number[k] = i;
                s.token[k] = a.tokens[d.first + i];
            }
            count += __popcll(m);
        }
        if (lane == 0) s.count = count;
    }
    __syncthreads();
    for (int j = int(threadIdx.x); j < s.count; j += int(blockDim.x)) {
        const int x = s.token[j];
        bool dull = x < 0 || x >= a.vocab;
        for (int i = 0; i < j && !dull; ++i) dull = s.token[i] == x;
        s.dull[j] = dull;
    }
    __syncthreads();
}

// Their q factors: 1, or what is left of q without the tokens before.
template <int kType>
__device__ __forceinline__ void draft_factors(const VerifyArgs& a, const char* row, const Whole& q, double rate,
                                              const double* table, Children& s)
{
    for (int j = int(threadIdx.x); j < s.count; j += int(blockDim.x))
        s.left[j] = a.distinct && !s.dull[j] ? share(logit<kType>(row, s.token[j]), q.top, rate, 1.0 / q.sum, table) : 0.0;
    __syncthreads();
    if (threadIdx.x == 0) {
        double by = 1.0;
        for (int j = 0; j < s.count; ++j) {
            s.by[j] = by;
            const double gone = s.left[j] * by;
            if (gone < 1.0) by /= 1.0 - gone;
        }
    }
    __syncthreads();
}

// The sum over a workgroup, the same for all threads and in every run.
template <int kThreads>
__device__ __forceinline__ double group_sum(double x, double* s_part)
{
    x = wave_sum(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s_part[threadIdx.x >> 6] = x;
    __syncthreads();
    double sum = 0.0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) sum += s_part[w];
    return sum;
}

// What child j's token has more than rest(p, q, upto), its B having ended with by(j).
template <int kType>
__device__ __forceinline__ double own_token(const char* pr, const char* qr, const Whole& p, const Whole& q, double rate,
                                            double ip, double iq, const double* table, const Children& s, int j, double upto)
{
    if (s.dull[j]) return 0.0;
    const double a = share(logit<kType>(pr, s.token[j]), p.top, rate, ip, table);
    const double b = share(logit<kType>(qr, s.token[j]), q.top, rate, iq, table);
    return rest(a, b, s.by[j]) - rest(a, b, upto);
}

// ---- siblings --------------------------------------------------------------------

// A workgroup per token with several children: what the refusal of each but the last leaves.
template <int kType>
__global__ void __launch_bounds__(kWalk) kvx_verify_siblings_kernel(const VerifyArgs a)
{
    __shared__ double s_table[kTable], s_part[kWalk / 64];
    __shared__ Children s_kids;
    const int row = int(blockIdx.x);
    const int r = request_at(a.starts, a.num_requests, row);
    if (r < 0 || r >= a.num_requests) return;
    const Drafts d = drafts_of(a, r);
    const int at = row - d.first;
    const double rate = rate_of(a, r);
    if (at >= d.n || rate == 0.0) return;
    fill_table(s_table);
    list_children(a, d, at, s_kids);
    const int count = s_kids.count;
    if (count < 2) return;
    const int lane = int(threadIdx.x) & 63;
    const Whole p = join(a.part[0] + int64_t(row) * a.parts, a.parts, rate, s_table, lane, 64);
    const Whole q = join(a.part[1] + int64_t(row) * a.parts, a.parts, rate, s_table, lane, 64);
    if (p.sum == 0.0 || q.sum == 0.0) return;
    const char* const pr = row_of(a, 0, row, kSize<kType>);
    const char* const qr = row_of(a, 1, row, kSize<kType>);
    constexpr int kV = kVec<kType>;
    // over both rows: each(l, l', v) for every token
    auto walk = [&](auto each) {
        for (int v = int(threadIdx.x) * kV; v < a.vocab; v += kWalk * kV) {
            if (v + kV <= a.vocab) {
                const u32x4 x = load16(pr + int64_t(v) * kSize<kType>), y = load16(qr + int64_t(v) * kSize<kType>);
#pragma unroll
                for (int e = 0; e < kV; ++e) each(element<kType>(x, e), element<kType>(y, e), v + e);
            } else {
                for (int e = v; e < a.vocab; ++e) each(logit<kType>(pr, e), logit<kType>(qr, e), e);
            }
        }
    };
    draft_factors<kType>(a, qr, q, rate, s_table, s_kids);
    const double ip = 1.0 / p.sum, iq = 1.0 / q.sum;
    double scale = 1.0, upto = 0.0;                    // A and B
    for (int k = 0; k + 1 < count; ++k) {
        upto += s_kids.by[k] / scale;
        double sum = 0.0;
        walk([&](float lp, float lq, int) {
            sum += rest(share(lp, p.top, rate, ip, s_table), share(lq, q.top, rate, iq, s_table), upto);
        });
        if (a.distinct)
            for (int j = int(threadIdx.x); j < k; j += kWalk) sum += own_token<kType>(pr, qr, p, q, rate, ip, iq, s_table, s_kids, j, upto);
        sum = group_sum<kWalk>(sum, s_part);
        const double left = sum > 0x1p-1000 ? 1.0 / (scale * sum) : 1.0;
        if (threadIdx.x == 0) {
            s_kids.by[k] = upto;
            a.left[d.first + s_kids.number[k]] = left;
        }
        scale *= left;
        __syncthreads();
    }
}

// ---- the next token ----------------------------------------------------------------

// The first v, in parts' order, for which the sum of the weights up to v is above `sample` times
// their whole; -1 where they sum to 0.  of_part(c) is a part's sum, weight(v) a token's; a
// workgroup of kWalk threads calls.
template <typename P, typename W>
__device__ __forceinline__ int draw(const VerifyArgs& a, float sample, double* s_scan, int* s_pick, P of_part, W weight)
{
    const int tid = int(threadIdx.x), lane = tid & 63, wave = tid >> 6;
    // sums of the threads before this one, and the whole
    auto scan = [&](double mine, double& whole) {
        double upto = mine;
        for (int o = 1; o < 64; o <<= 1) {
            const double u = __shfl_up(upto, o);
            if (lane >= o) upto += u;
        }
        __syncthreads();
        if (lane == 63) s_scan[wave] = upto;
        __syncthreads();
        double before = 0.0;
        whole = 0.0;
        for (int w = 0; w < kWalk / 64; ++w) {
            before += w < wave ? s_scan[w] : 0.0;
            whole += s_scan[w];
        }
        const double prev = __shfl_up(upto, 1);
        return before + (lane ? prev : 0.0);
    };
    const float cut = sample > 0.0f ? fminf(sample, 0x1.fffffep-1f) : 0.0f;
    // the part: consecutive ones to a thread, the first of them kept
    const int per = (a.parts + kWalk - 1) / kWalk, c0 = min(tid * per, a.parts), c1 = min(c0 + per, a.parts);
    const double own = c0 < c1 ? of_part(c0) : 0.0;
    double mine = own, whole;
    for (int c = c0 + 1; c < c1; ++c) mine += of_part(c);
    double before = scan(mine, whole);
    if (!(whole > 0.0)) return -1;
    double target = double(cut) * whole;
    // s_pick: the part, and the sum before it; should rounding leave none, the last that has a weight
    if (tid == 0) s_pick[0] = INT32_MAX, s_pick[1] = -1;
    __syncthreads();
    int found = INT32_MAX, some = -1;
    double at = before;
    for (int c = c0; c < c1; ++c) {
        const double x = c == c0 ? own : of_part(c);
        if (x > 0.0) some = c;
        at += x;
        if (x > 0.0 && at > target && found == INT32_MAX) found = c;
    }
    if (found != INT32_MAX) atomicMin(&s_pick[0], found);
    if (some >= 0) atomicMax(&s_pick[1], some);
    __syncthreads();
    const int part = s_pick[0] != INT32_MAX ? s_pick[0] : max(s_pick[1], 0);
    __syncthreads();
    if (part >= c0 && part < c1) {
        double sum = before;
        for (int c = c0; c < part; ++c) sum += c == c0 ? own : of_part(c);
        s_scan[kWalk / 64] = sum;
    }
    if (tid == 0) s_pick[0] = INT32_MAX, s_pick[1] = -1;
    __syncthreads();
    target -= s_scan[kWalk / 64];
    // the token: 8 consecutive ones to a thread
    constexpr int kEach = kPart / kWalk;
    double w[kEach], sum = 0.0;
    const int v0 = part * kPart + tid * kEach;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        w[e] = v0 + e < a.vocab ? weight(v0 + e) : 0.0;
        sum += w[e];
    }
    at = scan(sum, whole);
    found = INT32_MAX, some = -1;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        if (w[e] > 0.0) some = v0 + e;
        at += w[e];
        if (w[e] > 0.0 && at > target && found == INT32_MAX) found = v0 + e;
    }
    if (found != INT32_MAX) atomicMin(&s_pick[0], found);
    if (some >= 0) atomicMax(&s_pick[1], some);
    __syncthreads();
    return s_pick[0] != INT32_MAX ? s_pick[0] : s_pick[1];
}

// Without a draft: from p with the tokens of `refusal` at 0, or all of p where that leaves nothing.
template <int kType>
__device__ __forceinline__ int draw_plain(const VerifyArgs& a, const char* row, const Part* part, const Whole& p,
                                          double rate, const int* refusal, int count, float sample,
                                          const double* table, double* s_scan, int* s_pick)
{
    auto weight = [&](int v) { return share(logit<kType>(row, v), p.top, rate, 1.0, table); };
    auto of_part = [&](int c) {
        return part[c].top == -INFINITY ? 0.0 : part[c].sum * exp2_256th(table, (double(part[c].top) - double(p.top)) * rate);
    };
    for (;; count = 0) {
        const int next = draw(
            a, sample, s_scan, s_pick,
            [&](int c) {
                const double all = of_part(c);
                double x = all;
                for (int j = 0; j < count; ++j)
                    if (refusal[j] / kPart == c) x -= weight(refusal[j]);
                // what rounding leaves of a part whose weight was refused
                return x > 0x1p-40 * all ? x : 0.0;
            },
            [&](int v) {
                for (int j = 0; j < count; ++j)
                    if (refusal[j] == v) return 0.0;
                return weight(v);
            });
        if (next >= 0 || count == 0) return next;
    }
}

// ---- walk ------------------------------------------------------------------------

template <int kType, bool kDraft>
__global__ void __launch_bounds__(kWalk) kvx_verify_walk_kernel(const VerifyArgs a)
{
    __shared__ double s_table[kTable], s_scan[kWalk / 64 + 1];
    __shared__ Whole s_row[kDraft ? 2 : 1][kMaxDrafted];
    __shared__ int s_best[kMaxDrafted], s_parent[kMaxDrafted], s_token[kMaxDrafted], s_pick[2], s_last, s_leaf;
    __shared__ double s_own[kMaxDrafted], s_drafted[kDraft ? kMaxDrafted : 1];
    __shared__ uint8_t s_dull[kMaxDrafted];
    const int tid = int(threadIdx.x), r = int(blockIdx.x);
    const Drafts d = drafts_of(a, r);
    int32_t* const out = a.accepted + int64_t(r) * a.a_stride;
    if (d.n == 0) {
        for (int i = tid; i < a.a_stride; i += kWalk) out[i] = -1;
        if (tid == 0) {
            a.counts[r] = 0;
            a.next[r] = -1;
            if constexpr (kDraft) a.last[r] = -1;
        }
        return;
    }
    fill_table(s_table);
    const double rate = rate_of(a, r);
    // rows, as many lanes to each as it has parts
    int lanes = 1;
    while (lanes < 64 && lanes < a.parts) lanes <<= 1;
    __syncthreads();
    for (int side = 0; side < (kDraft ? 2 : 1); ++side)
        for (int i0 = 0; i0 < d.n; i0 += kWalk / lanes) {
            const int i = i0 + tid / lanes, lane = tid & (lanes - 1);
            const bool there = i < d.n;
            const Whole w = join(a.part[side] + int64_t(d.first + min(i, d.n - 1)) * a.parts, a.parts, rate, s_table,
                                 lane, lanes);
            if (there && lane == 0) s_row[side][i] = w;
        }
    for (int i = tid; i < d.n; i += kWalk) {
        s_best[i] = INT32_MAX;
        s_parent[i] = parent_of(a, d.first, i);
        s_token[i] = a.tokens[d.first + i];
    }
    __syncthreads();
    // every token's shares of its parent's rows, and whether an earlier sibling is the same token
    for (int i = 1 + tid; i < d.n; i += kWalk) {
        const int u = s_parent[i], x = s_token[i];
        bool dull = u < 0 || x < 0 || x >= a.vocab;
        double own = 0.0, drafted = 0.0;
        if (!dull && rate != 0.0) {
            const Whole p = s_row[0][u];
            if (p.sum != 0.0)
                own = share(logit<kType>(row_of(a, 0, d.first + u, kSize<kType>), x), p.top, rate, 1.0 / p.sum, s_table);
            if constexpr (kDraft) {
                const Whole q = s_row[1][u];
                if (q.sum != 0.0)
                    drafted = share(logit<kType>(row_of(a, 1, d.first + u, kSize<kType>), x), q.top, rate, 1.0 / q.sum,
                                    s_table);
            }
        }
        for (int j = u + 1; j < i && !dull && a.parents; ++j) dull = s_parent[j] == u && s_token[j] == x;
        s_own[i] = own;
        if constexpr (kDraft) s_drafted[i] = drafted;
        s_dull[i] = dull;
    }
    __syncthreads();
    // would its parent accept it, the siblings before it being refused?
    for (int i = 1 + tid; i < d.n; i += kWalk) {
        const int u = s_parent[i], x = s_token[i];
        if (u < 0 || x < 0 || x >= a.vocab || s_row[0][u].sum == 0.0) continue;
        bool yes;
        if (rate == 0.0) {
            yes = x == s_row[0][u].at;
        } else if constexpr (kDraft) {
            if (s_row[1][u].sum == 0.0) continue;
            double left = s_own[i], by = 1.0;
            bool gone = false;
            for (int j = u + 1; j < i && a.parents; ++j) {
                if (s_parent[j] != u) continue;
                left = fmax(left - (gone ? 0.0 : s_drafted[i] * by), 0.0) * a.left[d.first + j];
                if (!a.distinct) continue;
                gone |= x == s_token[j];
                const double off = s_dull[j] ? 0.0 : s_drafted[j] * by;
                if (off < 1.0) by /= 1.0 - off;
            }
            yes = double(a.uniforms[d.first + i]) * (gone ? 0.0 : s_drafted[i] * by) < left;
        } else {
            double left = 1.0;
            for (int j = u + 1; j < i && a.parents; ++j)
                if (s_parent[j] == u && !s_dull[j]) left -= s_own[j];
            yes = !s_dull[i] && double(a.uniforms[d.first + i]) * left < s_own[i];
        }
        if (yes) atomicMin(&s_best[u], i);
    }
    __syncthreads();
    if (tid == 0) {
        int node = 0, count = 0;
        for (;;) {
            out[count++] = node;
            if (count == a.a_stride || s_best[node] == INT32_MAX) break;
            node = s_best[node];
        }
        a.counts[r] = count;
        s_last = node;
        s_leaf = count == a.a_stride;
        s_pick[0] = count;
    }
    __syncthreads();
    for (int i = s_pick[0] + tid; i < a.a_stride; i += kWalk) out[i] = -1;
    const int last = s_last;
    const Whole p = s_row[0][last];
    if (p.sum == 0.0 || rate == 0.0) {
        if (tid == 0) {
            a.next[r] = p.sum == 0.0 ? -1 : p.at;
            if constexpr (kDraft) a.last[r] = -1;
        }
        return;
    }
    if constexpr (kDraft) {
        const bool leaf = s_leaf || s_row[1][last].sum == 0.0;
        if (tid == 0) a.last[r] = last | (leaf ? kLeaf : 0);
    } else {
        // the tokens refused there, each once
        int* const refusal = s_best;
        __syncthreads();
        if (tid < 64) {
            int count = 0;
            for (int i0 = last + 1; i0 < d.n && !s_leaf; i0 += 64) {
                const int i = i0 + tid;
                const bool mine = i < d.n && s_parent[i] == last && !s_dull[i];
                const uint64_t m = __ballot(mine);
                if (mine) refusal[count + __popcll(m & ((uint64_t(1) << tid) - 1))] = s_token[i];
                count += __popcll(m);
            }
            if (tid == 0) s_last = count;
        }
        __syncthreads();
        const int next = draw_plain<kType>(a, row_of(a, 0, d.first + last, kSize<kType>),
                                           a.part[0] + int64_t(d.first + last) * a.parts, p, rate, refusal, s_last,
                                           a.samples[r], s_table, s_scan, s_pick);
        if (tid == 0) a.next[r] = next;
    }
}

// ---- residual and draw ---------------------------------------------------------------

// What the last token's row is, and its children with their factors; false: nothing to draw.
template <int kType>
__device__ __forceinline__ bool last_row(const VerifyArgs& a, int r, double* table, Children& kids, Whole& p, Whole& q,
                                         int64_t& row, double& rate, int& count)
{
    const int mark = a.last[r];
    if (mark < 0) return false;
    fill_table(table);
    const int at = mark & ~kLeaf;
    const Drafts d = drafts_of(a, r);
    rate = rate_of(a, r);
    row = d.first + at;
    list_children(a, d, at, kids);
    const int lane = int(threadIdx.x) & 63;
    count = mark & kLeaf ? 0 : kids.count;
    p = join(a.part[0] + row * a.parts, a.parts, rate, table, lane, 64);
    if (count > 0) {
        q = join(a.part[1] + row * a.parts, a.parts, rate, table, lane, 64);
        draft_factors<kType>(a, row_of(a, 1, row, kSize<kType>), q, rate, table, kids);
        for (int j = int(threadIdx.x); j + 1 < count; j += int(blockDim.x)) kids.left[j] = a.left[d.first + kids.number[j]];
        __syncthreads();
        if (threadIdx.x == 0) {
            double scale = 1.0, upto = 0.0;
            for (int j = 0; j < count; ++j) {
                upto += kids.by[j] / scale;
                kids.by[j] = upto;
                if (j + 1 < count) scale *= kids.left[j];
            }
        }
    }
    __syncthreads();
    return true;
}

// A wave sums a part of r after the last token.
template <int kType>
__global__ void __launch_bounds__(kWg) kvx_verify_residual_kernel(const VerifyArgs a)
{
    constexpr int kV = kVec<kType>;
    __shared__ double s_table[kTable];
    __shared__ Children s_kids;
    const int groups = (a.parts + kWaves - 1) / kWaves;
    const int r = int(blockIdx.x) / groups, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
    const int c = (int(blockIdx.x) - r * groups) * kWaves + wave, lane = int(threadIdx.x) & 63;
    Whole p, q = {};
    int64_t row;
    double rate;
    int count;
    if (!last_row<kType>(a, r, s_table, s_kids, p, q, row, rate, count) || c >= a.parts) return;
    const int64_t from = int64_t(c) * kPart * kSize<kType>;
    const char* const x = row_of(a, 0, row, kSize<kType>) + from;
    const char* const y = row_of(a, 1, row, kSize<kType>) + from;
    const int n = min(kPart, a.vocab - c * kPart);
    double sum = 0.0;
    if (count == 0) {
        const Part t = a.part[0][row * a.parts + c];
        if (lane == 0 && t.top != -INFINITY)
            sum = t.sum * exp2_256th(s_table, (double(t.top) - double(p.top)) * rate);
    } else {
        const double ip = 1.0 / p.sum, iq = 1.0 / q.sum;
        // after the last refusal r needs no sum of 1
        const double upto = s_kids.by[count - 1];
        auto one = [&](float lp, float lq) {
            return rest(share(lp, p.top, rate, ip, s_table), share(lq, q.top, rate, iq, s_table), upto);
        };
        for (int v = lane * kV; v < n; v += 64 * kV) {
            if (v + kV <= n) {
                const u32x4 s = load16(x + v * kSize<kType>), t = load16(y + v * kSize<kType>);
#pragma unroll
                for (int e = 0; e < kV; ++e) sum += one(element<kType>(s, e), element<kType>(t, e));
            } else {
                for (int e = v; e < n; ++e) sum += one(logit<kType>(x, e), logit<kType>(y, e));
            }
        }
        if (a.distinct)
            for (int j = lane; j + 1 < count; j += 64)
                if (s_kids.token[j] / kPart == c)
                    sum += own_token<kType>(x - from, y - from, p, q, rate, ip, iq, s_table, s_kids, j, upto);
    }
    sum = wave_sum(sum);
    if (lane == 0) a.residual[int64_t(r) * a.parts + c] = sum;
}

template <int kType>
__global__ void __launch_bounds__(kWalk) kvx_verify_draw_kernel(const VerifyArgs a)
{
    __shared__ double s_table[kTable], s_scan[kWalk / 64 + 1];
    __shared__ int s_pick[2];
    __shared__ Children s_kids;
    const int r = int(blockIdx.x);
    Whole p, q = {};
    int64_t row;
    double rate;
    int count;
    if (!last_row<kType>(a, r, s_table, s_kids, p, q, row, rate, count)) return;
    const char* const x = row_of(a, 0, row, kSize<kType>);
    const char* const y = row_of(a, 1, row, kSize<kType>);
    const float sample = a.samples[r];
    const double ip = 1.0 / p.sum, iq = count ? 1.0 / q.sum : 0.0;
    int next = draw(
        a, sample, s_scan, s_pick, [&](int c) { return a.residual[int64_t(r) * a.parts + c]; },
        [&](int v) {
            if (count == 0) return share(logit<kType>(x, v), p.top, rate, 1.0, s_table);
            double upto = s_kids.by[count - 1];
            for (int j = 0; j < count && a.distinct; ++j)
                if (s_kids.token[j] == v) {
                    upto = s_kids.by[j];
                    break;
                }
            return rest(share(logit<kType>(x, v), p.top, rate, ip, s_table),
                        share(logit<kType>(y, v), q.top, rate, iq, s_table), upto);
        });
    if (next < 0)
        next = draw_plain<kType>(a, x, a.part[0] + row * a.parts, p, rate, s_kids.number, 0, sample, s_table, s_scan, s_pick);
    if (threadIdx.x == 0) a.next[r] = next;
}

// of all rows, the draft's too
int64_t part_groups(const VerifyArgs& a)
{
    return (int64_t(a.total_tokens) * a.parts * (a.draft ? 2 : 1) + kWaves - 1) / kWaves;
}

int64_t residual_groups(const VerifyArgs& a) { return int64_t(a.num_requests) * ((a.parts + kWaves - 1) / kWaves); }

template <int kType>
int go(const VerifyArgs& a, void* stream)
{
    const int64_t R = a.num_requests, N = a.total_tokens;
    int err = 0;
    if (N > 0) err = launch_kernel(kvx_verify_parts_kernel<kType>, part_groups(a), kWg, stream, a);
    if (!err && a.draft && a.parents && N > 0) err = launch_kernel(kvx_verify_siblings_kernel<kType>, N, kWalk, stream, a);
    if (err) return err;
    if (!a.draft) return launch_kernel(kvx_verify_walk_kernel<kType, false>, R, kWalk, stream, a);
    err = launch_kernel(kvx_verify_walk_kernel<kType, true>, R, kWalk, stream, a);
    if (!err) err = launch_kernel(kvx_verify_residual_kernel<kType>, residual_groups(a), kWg, stream, a);
    if (!err) err = launch_kernel(kvx_verify_draw_kernel<kType>, R, kWalk, stream, a);
    return err;
}

}  // namespace

double verify_threads(const VerifyArgs& a)
{
    double most = std::max(double(part_groups(a)) * kWg, double(a.num_requests) * kWalk);
    if (a.draft) most = std::max(most, double(residual_groups(a)) * kWg);
    if (a.draft && a.parents) most = std::max(most, double(a.total_tokens) * kWalk);
    return most;
}

int launch_verify(const VerifyArgs& a, int dtype, void* stream)
{
    switch (dtype) {
    case KVX_FP16: return go<kF16>(a, stream);
    case KVX_BF16: return go<kB16>(a, stream);
    default: return go<kF32>(a, stream);
    }
}

}  // namespace kvx
