// gfx950 kernels that write and move rows of the paged cache: kvx_append (the
// new tokens' rows, with rotary positions), kvx_evict (selection by weight) and
// the move of rows up their request, shared by kvx_evict and kvx_commit.
#include <hip/hip_runtime.h>

#include "kvx_ops_dev.h"

namespace kvx {
namespace {

constexpr int kWg = 256;

// ---- append ------------------------------------------------------------------

// Maximum over each aligned group of 2^lg lanes, lg <= 5.
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

// One workgroup per token.  The turns of its pairs (cosine and sine of the
// fp32 angle, reduced in fp64 to a fraction of a turn) are computed once into
// LDS and shared by its q_heads + Hd turned heads; a power-of-two group of
// lanes covers a head, 8 elements (16 bytes) a lane.
template <bool kBf16, int kCache>
__global__ void __launch_bounds__(kWg) kvx_append_kernel(const AppendArgs a)
{
    __shared__ float2 turn[128];
    const int t = int(blockIdx.x);
    const int D = a.c.dim, P = a.pairs;
    for (int i = threadIdx.x; i < P; i += kWg) {
        int axis = 0;
#pragma unroll
        for (int s = 0; s < 3; ++s) axis += i >= a.sec_end[s];
        const float pos = static_cast<float>(a.positions[int64_t(axis) * a.b.total_tokens + t]);
        const double turns = double(pos * a.inv_freq[i]) * 0.15915494309189533577;
        const float frac = static_cast<float>(turns - rint(turns));
        float sn, cs;
        sincospif(2.0f * frac, &sn, &cs);
        turn[i] = make_float2(cs, sn);
    }
    const int r = request_at(a.b.starts, a.c.num_requests, t);
    int64_t row = -1;
    if (r >= 0 && r < a.c.num_requests) {
        const Request rq = request_of(a.c, a.b, r);
        const int j = rq.ctx + (t - rq.first);
        if (t - rq.first < rq.n && j < rq.total) row = slot_row(a.c, r, j);
    }
    __syncthreads();
    const int per = 1 << a.lg_row;
    const int lane = int(threadIdx.x) & (per - 1), e0 = lane * 8;
    const int rows = a.q_heads + 2 * a.c.hd;
    for (int h0 = 0; h0 < rows; h0 += kWg >> a.lg_row) {
        const int h = h0 + (int(threadIdx.x) >> a.lg_row);
        const bool live = h < rows && e0 < D;
        const bool is_q = h < a.q_heads, is_v = h >= a.q_heads + a.c.hd;
        float x[8] = {};
        if (live) {
            const uint16_t* src = is_q ? a.q + t * a.q_stride + int64_t(h) * D
                                : is_v ? a.v + t * a.v_stride + int64_t(h - a.q_heads - a.c.hd) * D
                                       : a.k + t * a.k_stride + int64_t(h - a.q_heads) * D;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int i = e0 + e;
                x[e] = value16<kBf16>(src[i]);
                if (!is_v && i < 2 * P) {
                    int pair, other;
                    bool second;
                    if (a.interleaved) {
                        pair = i >> 1, second = i & 1, other = i ^ 1;
                    } else {
                        second = i >= P, pair = second ? i - P : i, other = second ? i - P : i + P;
                    }
                    const float y = value16<kBf16>(src[other]);
                    const float2 cs = turn[pair];
                    x[e] = second ? x[e] * cs.x + y * cs.y : x[e] * cs.x - y * cs.y;
                }
            }
        }
        // every lane has read its elements before q_out, which may be q, is written
        __syncthreads();
        if (is_q) {
            if (live) {
                uint16_t* dst = a.q_out + t * a.q_out_stride + int64_t(h) * D;
#pragma unroll
                for (int e = 0; e < 8; ++e) dst[e0 + e] = uint16_t(bits16<kBf16>(x[e]));
            }
            continue;
        }
        const int kv = is_v ? 1 : 0, head = h - a.q_heads - (is_v ? a.c.hd : 0);
        char* plane = a.c.base + kv * a.c.plane_bytes;
        if constexpr (kCache == KVX_FP16 || kCache == KVX_BF16) {
            if (live && row >= 0) {
                uint16_t* dst = reinterpret_cast<uint16_t*>(plane) + (row + head) * D;
#pragma unroll
                for (int e = 0; e < 8; ++e) dst[e0 + e] = uint16_t(bits16<kCache == KVX_BF16>(x[e]));
            }
        } else {
            constexpr bool kE5 = kCache == KVX_FP8_E5M2;
            float m = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) m = fmaxf(m, __builtin_fabsf(x[e]));  // a NaN takes no part
            m = lanes_max(m, a.lg_row);
            const float s = m / (kE5 ? 57344.0f : 448.0f);
            if (live && row >= 0) {
                uint8_t* dst = reinterpret_cast<uint8_t*>(plane) + (row + head) * D;
#pragma unroll
                for (int e = 0; e < 8; ++e) dst[e0 + e] = uint8_t(code8<kE5>(x[e], s));
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

// Inclusive sum over a workgroup of 256, in thread order, and the total.
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t* part, uint32_t& total)
{
    const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) >> 6;
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t u = __shfl_up(v, o);
        if (lane >= o) v += u;
    }
    __syncthreads();
    if (lane == 63) part[wave] = v;
    __syncthreads();
    uint32_t before = 0;
    total = 0;
#pragma unroll
    for (int k = 0; k < kWg / 64; ++k) {
        before += k < wave ? part[k] : 0u;
        total += part[k];
    }
    return v + before;
}

// One workgroup per (layer, request, head).  The weight of the last slot that
// stays is found by its key's four bytes, highest first: a histogram of the
// candidates that agree with the bytes found so far, walked from the top.  Then
// one pass in slot order writes what stays; of the slots that tie with that
// weight the first ones.
__global__ void __launch_bounds__(kWg) kvx_select_kernel(const EvictArgs a)
{
    __shared__ uint32_t hist[256];
    __shared__ uint32_t part[kWg / 64];
    __shared__ uint32_t s_byte, s_left;
    const int lrh = int(blockIdx.x);
    const int r = (lrh / a.c.hd) % a.c.num_requests;
    const int T = min(min(max(a.lens[r], 0), a.max_len), a.c.row_slots);
    const int keep = min(T, a.budget);
    const float* w = a.weights + int64_t(lrh) * a.w_stride;
    float* w_out = a.weights_out + int64_t(lrh) * a.w_stride;
    int32_t* kept = a.kept + int64_t(lrh) * a.budget;
    if (lrh < a.c.num_requests * a.c.hd && lrh % a.c.hd == 0 && threadIdx.x == 0)
        a.new_lens[r] = keep;
    if (T <= a.budget) {
        for (int i = threadIdx.x; i < a.budget; i += kWg) {
            if (i < T && w_out != w) w_out[i] = w[i];
            kept[i] = i < T ? i : -1;
        }
        return;
    }
    const int lo = a.sink, hi = T - a.recent;    // candidates; sink + recent <= budget < T
    uint32_t left = uint32_t(a.budget - a.sink - a.recent);
    uint32_t key = 0;                            // bytes found so far
    if (left) {
        for (int shift = 24; shift >= 0; shift -= 8) {
            hist[threadIdx.x] = 0;
            __syncthreads();
            for (int j = lo + int(threadIdx.x); j < hi; j += kWg) {
                const uint32_t k = weight_key(w[j]);
                if (shift == 24 || (k >> (shift + 8)) == (key >> (shift + 8)))
                    atomicAdd(&hist[(k >> shift) & 255u], 1u);
            }
            __syncthreads();
            // thread i holds byte 255 - i: the inclusive sum counts the larger ones too
            const uint32_t mine = hist[255 - threadIdx.x];
            uint32_t total;
            const uint32_t upto = block_scan(mine, part, total);
            if (upto >= left && upto - mine < left) {
                s_byte = 255u - threadIdx.x;
                s_left = left - (upto - mine);
            }
            __syncthreads();
            key |= s_byte << shift;
            left = s_left;
            __syncthreads();
        }
    }
    // `left` slots of weight `key` stay, and all above it
    const bool any = a.budget > a.sink + a.recent;
    uint32_t ties = 0, out = 0;
    for (int j0 = 0; j0 < T; j0 += kWg) {
        const int j = j0 + int(threadIdx.x);
        const float x = j < T ? w[j] : 0.0f;
        const bool cand = j >= lo && j < hi;
        const uint32_t k = weight_key(x);
        const bool tie = any && cand && k == key;
        uint32_t n_ties, n_out;
        const uint32_t rank = block_scan(tie ? 1u : 0u, part, n_ties) + ties;
        const bool stay = j < T && (!cand || (any && k > key) || (tie && rank <= left));
        const uint32_t at = block_scan(stay ? 1u : 0u, part, n_out) + out;
        // w_out may be w: position at - 1 <= j, and every thread has read its weight
        if (stay) {
            kept[at - 1] = j;
            w_out[at - 1] = x;
        }
        ties += n_ties;
        out += n_out;
    }
}

// ---- rows move up -------------------------------------------------------------

// One workgroup per (layer, k/v, request, head) moves its rows in order, a
// group of rows at a time: all of a group's rows are read, then written.  A row
// never moves down (index[i] >= i), so a write can only hit rows that this or
// an earlier group has read.
template <bool kCommit>
__global__ void __launch_bounds__(kWg) kvx_move_kernel(const MoveArgs a)
{
    const int H = a.c.hd, R = a.c.num_requests;
    int u = int(blockIdx.x);
    const int h = u % H;
    u /= H;
    const int r = u % R;
    u /= R;
    const int kv = u & 1, layer = u >> 1;
    int rows, first = 0;
    const int32_t* index;
    if constexpr (kCommit) {
        first = max(a.contexts[r], 0);
        rows = min(a.new_lens[r] - first, a.stride);
        index = a.index + int64_t(r) * a.stride;
    } else {
        const int T = min(min(max(a.lens[r], 0), a.max_len), a.c.row_slots);
        rows = T > a.stride ? a.stride : 0;
        index = a.index + ((int64_t(layer) * R + r) * H + h) * a.stride;
    }
    const int64_t plane = int64_t(2) * layer + kv;
    char* base = a.c.base + plane * a.c.plane_bytes;
    float* scales = a.c.scales ? a.c.scales + plane * a.c.plane_scales : nullptr;
    const int chunks = a.c.row_bytes >> 4;                 // 16-byte pieces of a row
    int lg = 0;
    while ((1 << lg) < chunks) ++lg;
    const int per = 1 << lg, group = kWg >> lg;
    const int piece = int(threadIdx.x) & (per - 1);
    for (int i0 = 0; i0 < rows; i0 += group) {
        const int i = i0 + (int(threadIdx.x) >> lg);
        int64_t src = -1, dst = -1;
        uint4 x = make_uint4(0, 0, 0, 0);
        float s = 0.0f;
        if (i < rows && piece < chunks) {
            const int from = index[i];
            if (from > i && first + from < a.c.row_slots) {
                src = slot_row(a.c, r, first + from);
                dst = slot_row(a.c, r, first + i);
            }
            if (src < 0) dst = -1;
        }
        if (dst >= 0) {
            x = *reinterpret_cast<const uint4*>(base + (src + h) * a.c.row_bytes + piece * 16);
            if (scales && piece == 0) s = scales[src + h];
        }
        __builtin_amdgcn_s_waitcnt(0);                     // this group's rows are in registers
        __syncthreads();
        if (dst >= 0) {
            *reinterpret_cast<uint4*>(base + (dst + h) * a.c.row_bytes + piece * 16) = x;
            if (scales && piece == 0) scales[dst + h] = s;
        }
    }
}

// The accepted paths' lengths: entries ascend strictly and their slots lie in
// the block-table row; the first that does not ends the path.
__global__ void __launch_bounds__(kWg) kvx_path_kernel(const CacheArgs c, const CommitArgs a)
{
    const int r = int(blockIdx.x) * kWg + int(threadIdx.x);
    if (r >= c.num_requests) return;
    const int first = max(a.contexts[r], 0);
    const int most = min(a.counts[r], a.a_stride);
    int n = 0, before = -1;
    while (n < most) {
        const int e = a.accepted[int64_t(r) * a.a_stride + n];
        if (e <= before || int64_t(first) + e >= c.row_slots) break;
        before = e;
        ++n;
    }
    a.new_lens[r] = first + n;
}

int done() { return int(hipGetLastError()); }

template <typename K, typename A>
int run(K kernel, int64_t grid, const A& args, void* stream)
{
    kernel<<<dim3(uint32_t(grid)), dim3(kWg), 0, static_cast<hipStream_t>(stream)>>>(args);
    return done();
}

template <bool kBf16>
int append_as(const AppendArgs& a, int cache_dtype, void* stream)
{
    const int64_t n = a.b.total_tokens;
    switch (cache_dtype) {
    case KVX_FP16: return run(kvx_append_kernel<kBf16, KVX_FP16>, n, a, stream);
    case KVX_BF16: return run(kvx_append_kernel<kBf16, KVX_BF16>, n, a, stream);
    case KVX_FP8_E4M3FN: return run(kvx_append_kernel<kBf16, KVX_FP8_E4M3FN>, n, a, stream);
    default: return run(kvx_append_kernel<kBf16, KVX_FP8_E5M2>, n, a, stream);
    }
}

}  // namespace

int launch_append(const AppendArgs& a, int dtype, int cache_dtype, void* stream)
{
    return dtype == KVX_BF16 ? append_as<true>(a, cache_dtype, stream)
                             : append_as<false>(a, cache_dtype, stream);
}

int launch_evict(const EvictArgs& a, int num_layers, void* stream)
{
    const int64_t units = int64_t(num_layers) * a.c.num_requests * a.c.hd;
    const int err = run(kvx_select_kernel, units, a, stream);
    if (err) return err;
    MoveArgs m = {};
    m.c = a.c;
    m.index = a.kept;
    m.stride = a.budget;
    m.num_layers = num_layers;
    m.lens = a.lens;
    m.max_len = a.max_len;
    return run(kvx_move_kernel<false>, 2 * units, m, stream);
}

int launch_commit(const CacheArgs& c, const CommitArgs& a, int num_layers, void* stream)
{
    kvx_path_kernel<<<dim3((c.num_requests + kWg - 1) / kWg), dim3(kWg), 0,
                      static_cast<hipStream_t>(stream)>>>(c, a);
    const int err = done();
    if (err || num_layers == 0 || a.a_stride == 0) return err;
    MoveArgs m = {};
    m.c = c;
    m.index = a.accepted;
    m.stride = a.a_stride;
    m.num_layers = num_layers;
    m.contexts = a.contexts;
    m.new_lens = a.new_lens;
    return run(kvx_move_kernel<true>, int64_t(2) * num_layers * c.num_requests * c.hd, m, stream);
}

}  // namespace kvx
