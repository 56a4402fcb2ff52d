// Device helpers of the decode operators: places in the paged cache, the
// requests of a batch, element types.
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

#include "kvx_ops_internal.h"

namespace kvx {

// Enqueues `kernel` and returns this launch's hipError_t (an earlier call's error
// is not taken for it).
template <typename... P>
int launch_kernel(void (*kernel)(P...), int64_t grid, int threads, void* stream,
                  const std::common_type_t<P>&... p)
{
    void* args[] = {const_cast<void*>(static_cast<const void*>(&p))...};
    return int(hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3(uint32_t(grid)),
                               dim3(uint32_t(threads)), args, 0, static_cast<hipStream_t>(stream)));
}

__device__ __forceinline__ uint32_t fast_div(uint32_t n, FastDiv d)
{
    return uint32_t((uint64_t(__umulhi(n, d.mul)) + n) >> d.shift);
}

// Row index ((page x block_size + slot) x hd) of slot j of request r in a
// plane, or -1 where its page id names no page.  j is below row_slots.
__device__ __forceinline__ int64_t slot_row(const CacheArgs& c, int r, int j)
{
    const uint32_t blk = fast_div(uint32_t(j), c.div_bs);
    const int32_t page = c.table[int64_t(r) * c.bt_stride + blk];
    if (page < 0 || page >= c.num_blocks) return -1;
    return (int64_t(page) * c.block_size + (uint32_t(j) - blk * uint32_t(c.block_size))) * c.hd;
}

// The new tokens of request r, cut to the host's bounds: first token on the
// flat axis, their number, slots in use before them and in all.
struct Request {
    int32_t first, n, ctx, total;
};

__device__ __forceinline__ Request request_of(const CacheArgs& c, const BatchArgs& b, int r)
{
    Request q;
    const int32_t most = min(b.max_context, c.row_slots);
    const int32_t s0 = min(max(b.starts[r], 0), b.total_tokens);
    const int32_t s1 = min(max(b.starts[r + 1], s0), b.total_tokens);
    q.first = s0;
    q.n = min(s1 - s0, b.max_tokens);
    q.ctx = min(max(b.contexts[r], 0), most);
    q.total = min(q.ctx + q.n, most);
    return q;
}

// The request that token t of the flat axis belongs to: the last r with
// starts[r] <= t (a wave counts the starts, 64 at a time).
__device__ __forceinline__ int request_at(const int32_t* starts, int num_requests, int t)
{
    const int lane = int(threadIdx.x) & 63;
    int r = -1;
    for (int base = 0; base <= num_requests; base += 64) {
        const bool le = base + lane <= num_requests && starts[base + lane] <= t;
        const uint64_t m = __ballot(le);
        r += __popcll(m);
        if (m != ~uint64_t(0)) break;
    }
    return r;
}

__device__ __forceinline__ float f16_value(uint32_t h)
{
    return static_cast<float>(__builtin_bit_cast(_Float16, static_cast<unsigned short>(h)));
}

// 16-bit bits -> fp32, exactly
template <bool kBf16>
__device__ __forceinline__ float value16(uint32_t h)
{
    return kBf16 ? __uint_as_float(h << 16) : f16_value(h);
}

// fp32 -> 16-bit bits, to nearest even
template <bool kBf16>
__device__ __forceinline__ uint32_t bits16(float x)
{
    if constexpr (kBf16)
        return __builtin_bit_cast(unsigned short, static_cast<__bf16>(x));
    else
        return __builtin_bit_cast(unsigned short, static_cast<_Float16>(x));
}

}  // namespace kvx
