// Device helpers shared by the attention kernels and the weights' kernel:
// matrix instructions, 8-bit codes widened to the queries' type, visibility as
// bit masks, scores.
//
// Scores are kept in units of log2: x2 = x log2(e), so that exp(x - m) is one
// v_exp_f32.  All products are formed transposed, S^T = K Q^T and O^T = V^T P^T:
// the accumulator then has one query row per lane column, a row's statistics and
// rescaling stay in its lanes, and the exponentials leave the registers in the
// order in which the second product takes them.
#pragma once

#include "kvx_ops_dev.h"

namespace kvx {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

enum Codes : int { kCodes16 = 0, kCodesE4m3 = 1, kCodesE5m2 = 2, kCodesE2m1 = 3 };

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <bool kBf16>
__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c)
{
    if constexpr (kBf16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                       __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a),
                                                      __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

template <bool kBf16>
__device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c)
{
    if constexpr (kBf16)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                       __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a),
                                                      __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// two fp32 values -> 16-bit pair, to nearest even
template <bool kBf16>
__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    const f32x2 v = {a, b};
    if constexpr (kBf16)
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
    else
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
}

// bytes 0-1 (kHi false) or 2-3 of a dword of codes -> a pair in the queries'
// type.  Every e4m3fn and e5m2 value is exact in bf16 and in fp16.
template <bool kBf16, int kCodes, bool kHi>
__device__ __forceinline__ uint32_t widen2(uint32_t w)
{
    if constexpr (kCodes == kCodesE4m3) {
        if constexpr (kBf16)
            return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, kHi));
        else
            return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, kHi));
    } else {
        if constexpr (kBf16)
            return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, 1.0f, kHi));
        else
            return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_bf8(w, 1.0f, kHi));
    }
}

// 8 codes -> 8 values in the queries' type
template <bool kBf16, int kCodes>
__device__ __forceinline__ u32x4 widen8(uint32_t lo, uint32_t hi)
{
    return u32x4{widen2<kBf16, kCodes, false>(lo), widen2<kBf16, kCodes, true>(lo),
                 widen2<kBf16, kCodes, false>(hi), widen2<kBf16, kCodes, true>(hi)};
}

// Codes of 4 bits are values of bf16 exactly, their group's scale in them: over such a
// cache products are bf16, and fp16 queries (and their weights) are taken as two bf16
// terms, which hold their 11 bits.
template <bool kBf16, int kCodes>
constexpr bool kMathBf16 = kBf16 || kCodes == kCodesE2m1;

// the factor of a group whose scale byte is b; NaN for the bytes that stand for none
__device__ __forceinline__ float group_factor(uint32_t b) { return __uint_as_float((b > 252u ? 255u : b) << 23); }

// byte kByte of a dword of 4-bit codes -> a pair of bf16
template <int kByte>
__device__ __forceinline__ uint32_t widen4(uint32_t w, float scale)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, kByte));
}

// 8 codes of 4 bits -> 8 bf16 values
__device__ __forceinline__ u32x4 widen4x8(uint32_t w, float scale)
{
    return u32x4{widen4<0>(w, scale), widen4<1>(w, scale), widen4<2>(w, scale), widen4<3>(w, scale)};
}

// an fp16 pair as two pairs of bf16 that sum to it (an infinity is its first alone)
__device__ __forceinline__ uint32_t two_terms(uint32_t h, uint32_t& rest)
{
    const float a = value16<false>(h & 0xFFFFu), b = value16<false>(h >> 16);
    const uint32_t w = pack2<true>(a, b);
    rest = pack2<true>(__builtin_fabsf(a) < INFINITY ? a - value16<true>(w & 0xFFFFu) : 0.0f,
                       __builtin_fabsf(b) < INFINITY ? b - value16<true>(w >> 16) : 0.0f);
    return w;
}

// Half `hi` (elements 2w, 2w + 1 of a row) of two keys -> their pair
template <bool kHi>
__device__ __forceinline__ uint32_t pair16(uint32_t key0, uint32_t key1)
{
    return __builtin_amdgcn_perm(key1, key0, kHi ? 0x07060302u : 0x05040100u);
}

// A value that the compiler does not know: what follows from it is formed where it is
// used.  After a walk over the slots the lane's place is taken from one, since what
// is formed ahead and kept until then costs the walk registers.
__device__ __forceinline__ int hidden(int x)
{
    __asm__ volatile("" : "+v"(x));
    return x;
}

// ---- non-finite values ---------------------------------------------------------
//
// A weight of 0 does not hide an infinity from a matrix product (0 x inf is
// NaN), whether the slot is not seen or its weight came to 0.  Where a tile is not
// seen whole by every row, the product takes its finite values only.  If there were
// others, or a sum of a tile seen whole is not finite, a second walk finds by three
// products of ones with the rows' visibility which sums have +inf, -inf or NaN
// among their terms, and these become that.

template <bool kBf16>
constexpr uint32_t kOne = kBf16 ? 0x3F80u : 0x3C00u;

// Non-zero when a word of elements or codes holds one that is not finite: the
// exponent (e4m3fn: all of the magnitude) is all ones exactly when adding its
// lowest bit carries into the sign's place; no carry leaves the element.
template <bool kBf16, int kCodes>
__device__ __forceinline__ uint32_t nonfinite(uint32_t w)
{
    if constexpr (kCodes == kCodesE4m3) return ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
    if constexpr (kCodes == kCodesE5m2) return ((w & 0x7C7C7C7Cu) + 0x04040404u) & 0x80808080u;
    return kBf16 ? ((w & 0x7F807F80u) + 0x00800080u) & 0x80008000u
                 : ((w & 0x7C007C00u) + 0x04000400u) & 0x80008000u;
}

// a word with its elements or codes that are not finite as 0
template <int kCodes>
__device__ __forceinline__ uint32_t without(uint32_t w, uint32_t found)
{
    return w & ~(kCodes == kCodes16 ? (found >> 15) * 0xFFFFu : (found >> 7) * 0xFFu);
}

// kind 0: finite values kept, others 0; 1: one where +inf; 2: -inf; 3: NaN
template <bool kBf16>
__device__ __forceinline__ uint32_t classify2(uint32_t w, int kind)
{
    constexpr uint32_t e = kBf16 ? 0x7F80u : 0x7C00u;
    uint32_t out = 0;
#pragma unroll
    for (int s = 0; s < 32; s += 16) {
        const uint32_t h = (w >> s) & 0xFFFFu, mag = h & 0x7FFFu;
        const int k = (mag & e) != e ? 0 : mag > e ? 3 : h >> 15 ? 2 : 1;
        out |= (k != kind ? 0u : kind == 0 ? h : kOne<kBf16>) << s;
    }
    return out;
}

template <bool kBf16>
__device__ __forceinline__ u32x4 classify8(u32x4 v, int kind)
{
    return u32x4{classify2<kBf16>(v.x, kind), classify2<kBf16>(v.y, kind),
                 classify2<kBf16>(v.z, kind), classify2<kBf16>(v.w, kind)};
}

// an 8-bit slot's scale as its codes that are not finite take it, and all of its
// codes where it is not finite itself: 1, -1, 0, +-inf or NaN
__device__ __forceinline__ float scale_kind(float s)
{
    return s == 0.0f || !(__builtin_fabsf(s) < INFINITY) ? s : __builtin_copysignf(1.0f, s);
}

// a pair times a factor each
template <bool kBf16>
__device__ __forceinline__ uint32_t times2(uint32_t w, float lo, float hi)
{
    return bits16<kBf16>(value16<kBf16>(w & 0xFFFFu) * lo) | bits16<kBf16>(value16<kBf16>(w >> 16) * hi) << 16;
}

// a sum by its weight in a join; one that is not finite stays so where the weight came to 0
__device__ __forceinline__ float weighted(float x, float w)
{
    return w != 0.0f ? x * w : __builtin_fabsf(x) < INFINITY ? 0.0f : x;
}

// whether one of kT vectors of kN sums is not finite (four chains, not one)
template <int kN, int kT>
__device__ __forceinline__ bool any_endless(const float __attribute__((ext_vector_type(kN))) (&o)[kT])
{
    float zero[4] = {};
#pragma unroll
    for (int t = 0; t < kT; ++t)
#pragma unroll
        for (int i = 0; i < kN; ++i) zero[i & 3] = __builtin_fmaf(o[t][i], 0.0f, zero[i & 3]);
    const float sum = (zero[0] + zero[1]) + (zero[2] + zero[3]);
    return sum != sum;
}

// Which of a lane's kN sums have such values among their terms, a bit a sum and kind.
template <int kN>
struct Had {
    uint64_t bits[3][(kN + 63) / 64] = {};
    __device__ __forceinline__ void add(int at, float count, int kind)
    {
        // no index by kind or place: the bits stay in registers
        const uint64_t bit = uint64_t(count > 0.0f) << (at & 63);
#pragma unroll
        for (int k = 0; k < 3; ++k)
#pragma unroll
            for (int w = 0; w < (kN + 63) / 64; ++w) bits[k][w] |= kind == k + 1 && at >> 6 == w ? bit : 0;
    }
    // what sum `at` is, which the products say is `o`
    __device__ __forceinline__ float of(int at, float o) const
    {
        const int w = kN <= 64 ? 0 : at >> 6, s = at & 63;
        const bool up = bits[0][w] >> s & 1, down = bits[1][w] >> s & 1, none = bits[2][w] >> s & 1;
        return none || (up && down) ? NAN : up ? INFINITY : down ? -INFINITY : o;
    }
};

// ---- visibility ------------------------------------------------------------------

__device__ __forceinline__ uint64_t low_bits(int n)  // n cut to 0 .. 64
{
    return n <= 0 ? 0 : n >= 64 ? ~uint64_t(0) : (uint64_t(1) << n) - 1;
}

// What tokens [i0, i1] of a request see: slots [0, pre) and [lo, hi), both
// starting at multiples of 64, numbered through as 0 .. len; slots [all_lo,
// all_hi) are seen by all of them.  Uniform over the wave.
struct Range {
    int pre, lo, len, hi, all_lo, all_hi;
    __device__ __forceinline__ int slot(int v) const { return v < pre ? v : v - pre + lo; }
};

__device__ __forceinline__ Range range_of(const AttendArgs& a, const Request& rq, int r, int i0, int i1)
{
    const int fix = a.prefix ? min(max(a.prefix[r], 0), rq.total) : 0;
    Range g;
    g.hi = a.b.tree ? rq.total : min(rq.total, max(rq.ctx + i1 + 1, fix));
    g.all_hi = a.b.tree ? rq.ctx : rq.ctx + i0 + 1;
    g.pre = g.lo = g.all_lo = 0;
    if (a.window > 0) {
        int first = rq.ctx + i0, last = rq.ctx + i1;
        if (a.b.positions) {
            first = INT32_MAX;
            last = INT32_MIN;
            for (int i = i0 + (int(threadIdx.x) & 63); i <= i1; i += 64) {
                const int p = a.b.positions[rq.first + i];
                first = min(first, p);
                last = max(last, p);
            }
            for (int s = 32; s; s >>= 1) {
                first = min(first, __shfl_xor(first, s));
                last = max(last, __shfl_xor(last, s));
            }
            first = __builtin_amdgcn_readfirstlane(first);
            last = __builtin_amdgcn_readfirstlane(last);
            // new tokens' slots may lie at any position: they are in the range, unseen whole
            g.all_hi = min(g.all_hi, rq.ctx);
        }
        // positions may be anything: differences in 64 bits, cut to the slots there are; given
        // ones say nothing about where the new tokens' slots begin to be seen
        const int64_t lo = max(int64_t(0), min(int64_t(first) - a.window + 1,
                                               int64_t(a.b.positions ? rq.ctx : rq.total)));
        g.all_lo = int(max(int64_t(0), min(int64_t(last) - a.window + 1, int64_t(INT32_MAX))));
        g.pre = (fix + 63) & ~63;
        g.lo = max(int(lo) & ~63, g.pre);
        if (g.pre >= g.hi) g.pre = 0, g.lo = 0;
    }
    g.len = g.pre + max(0, g.hi - g.lo);
    return g;
}

// The position of slot j.
__device__ __forceinline__ int place_of(const AttendArgs& a, const Request& rq, int j)
{
    return a.b.positions && j >= rq.ctx && j < rq.total ? a.b.positions[rq.first + j - rq.ctx] : j;
}

// Which of the 64 slots from j0 on a token sees; valid: those that lie in a
// page.
__device__ __forceinline__ uint64_t seen_of(const AttendArgs& a, const Request& rq, int r, int i, int qp,
                                            int j0, uint64_t valid)
{
    uint64_t m;
    if (!a.b.tree) {
        m = low_bits(rq.ctx + i + 1 - j0);
    } else {
        m = low_bits(rq.ctx - j0);
        if (j0 + 64 > rq.ctx) {
            const uint64_t* w = a.b.tree + int64_t(rq.first + i) * a.b.tree_stride;
            const int k = j0 - rq.ctx;              // -63 or more
            if (k < 0) {
                m |= w[0] << -k;
            } else {
                const int at = k >> 6, s = k & 63;
                uint64_t bits = at < a.b.tree_stride ? w[at] >> s : 0;
                if (s && at + 1 < a.b.tree_stride) bits |= w[at + 1] << (64 - s);
                m |= bits;
            }
        }
    }
    if (a.window > 0) {
        const int64_t lo = int64_t(qp) - a.window + 1 - j0;  // first slot of the window
        const uint64_t out = low_bits(int(max(int64_t(0), min(lo, int64_t(64)))));
        if (!a.b.positions || j0 + 64 <= rq.ctx) {
            m &= ~out;
        } else {
            const uint64_t old = low_bits(rq.ctx - j0);
            m &= ~(out & old);
            for (int k = max(0, rq.ctx - j0); k < min(64, rq.total - j0); ++k)
                if (int64_t(qp) - place_of(a, rq, j0 + k) >= a.window) m &= ~(uint64_t(1) << k);
        }
    }
    if (a.prefix) m |= low_bits(max(a.prefix[r], 0) - j0);
    return m & low_bits(rq.total - j0) & valid;
}

// ---- scores -----------------------------------------------------------------------

struct ScoreArgs {
    float c2;        // scale log2(e)
    float to_cap;    // scale 2 log2(e) / softcap: tanh by exp2
    float cap2;      // softcap log2(e)
    float by_cap;    // 1 / softcap
};

// What scores are beside the product: nothing (and a positive scale); biased, capped
// or of another scale; those with a cap above kWideCap.
enum Scores : int { kPlain = 0, kGeneral = 1, kWide = 2 };

// Caps up to here take tanh in the form whose error is absolute, 2^-22 of the cap: in
// units of the score no more than 1.5e-5, below a weight's own rounding.  Larger
// ones take another, in kernels of their own: beside it in the same ones it costs the
// smaller caps registers (weights of a prompt's last 32 tokens 69 us, 62 apart; trees
// over an fp8 cache 349, 337).
constexpr float kWideCap = 64.0f;

inline Scores scores_of(const AttendArgs& a)
{
    return a.softcap > kWideCap ? kWide : a.softcap > 0.0f || a.slopes || !(a.scale > 0.0f) ? kGeneral : kPlain;
}

__device__ __forceinline__ ScoreArgs score_args(const AttendArgs& a)
{
    constexpr float kMost = 3.402823466e38f;
    ScoreArgs s;
    s.c2 = a.scale * kLog2e;
    // finite also for the smallest caps: a score of 0 stays 0
    s.to_cap = a.softcap > 0.0f ? fmaxf(fminf(a.scale * (2.0f * kLog2e) / a.softcap, kMost), -kMost) : 0.0f;
    s.cap2 = a.softcap > 0.0f ? a.softcap * kLog2e : 0.0f;
    s.by_cap = a.softcap > 0.0f ? 1.0f / a.softcap : 0.0f;
    return s;
}

// softcap tanh(y) in units of log2, plus `more`; e2y is y 2 log2(e):
// tanh(y) = 1 - 2 / (exp(2 y) + 1).
__device__ __forceinline__ float capped(const ScoreArgs& s, float e2y, float more)
{
    return __builtin_fmaf(-2.0f * s.cap2, __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(e2y) + 1.0f),
                          s.cap2 + more);
}

// The same from the score x2 for any cap: an error of 2^-20 of the score.  Up to
// |y| = 1/4 the series of tanh, whose next term is 2^-21 of y there.
__device__ __forceinline__ float capped_wide(const ScoreArgs& s, float x2, float more)
{
    const float y = x2 * (kLn2 * s.by_cap), z = y * y;
    const float near = x2 * __builtin_fmaf(-z, __builtin_fmaf(-z, __builtin_fmaf(-z, 17.0f / 315.0f, 2.0f / 15.0f),
                                                              1.0f / 3.0f), 1.0f);
    return __builtin_fabsf(y) < 0.25f ? near + more : capped(s, x2 * (2.0f * s.by_cap), more);
}

// The product's x2, capped and biased; slope2 is the head's slope log2(e).
template <int kScores>
__device__ __forceinline__ float general_score(const ScoreArgs& s, float dot, float slope2, int distance)
{
    const float x = kScores == kWide ? capped_wide(s, dot * s.c2, 0.0f)
                    : s.cap2 > 0.0f  ? capped(s, dot * s.to_cap, 0.0f)
                                     : dot * s.c2;
    return x - slope2 * static_cast<float>(distance < 0 ? -distance : distance);
}

// Weights are formed as 2^kShift exp(x - m): an fp16 weight then keeps its 11
// bits down to 2^-20 of the row's largest.  The shift cancels in the quotient.
template <bool kBf16>
constexpr float kShift = kBf16 ? 0.0f : 6.0f;
// What stands for the reference of a sum of weights l: -inf where l is 0 (nothing
// seen) and NaN where l is NaN, since m, a maximum, passes NaN by.  The sums of
// waves and of splits are joined by it.
__device__ __forceinline__ float reference_of(float m, float l)
{
    return l == 0.0f ? -INFINITY : l != l ? l : m;
}
// A row's reference m is moved only when a score passes it by more than this:
// weights stay below 2^(kSlack + kShift), far inside both types.
constexpr float kSlack = 8.0f;

// fp16 weights over 8-bit codes.  What is rounded is a weight times its slot's
// scale, and scales may lie any number of powers of two apart.  Each row takes
// these products 2^lift times as large, so that the largest of them so far lies
// between 2^kLiftTop and 2^kLiftMost: those down to 2^-25 of it keep their 11 bits.
// lift falls when a product would pass 2^kLiftMost; when the reference m rises by
// d, lift rises by d as well and the sums of V stay as they are, so that what the
// new reference has made small does not keep the others down.  Only slots that the
// row sees count.  The weights themselves are formed 2^kLiftShift times smaller
// there: no product with a finite scale overflows.
constexpr float kLiftTop = 11.0f, kLiftMost = 15.0f, kLiftMax = 126.0f, kLiftShift = 16.0f;

// the lift of a row whose largest product, not yet lifted, is `most`
__device__ __forceinline__ float lift_of(float lift, float most)
{
    return most > 0.0f ? fminf(lift, kLiftTop - __builtin_amdgcn_logf(most)) : lift;
}

// what brings a row's sums of V back
__device__ __forceinline__ float unlifted(float lift, float more = 0.0f)
{
    return __builtin_amdgcn_exp2f(fminf(kLiftShift - lift + more, 127.0f));
}

// |x| where it is finite, else 0
__device__ __forceinline__ float finite_size(float x)
{
    const float a = __builtin_fabsf(x);
    return a < INFINITY ? a : 0.0f;
}

}  // namespace kvx
