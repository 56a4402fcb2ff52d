// Host side of kvx_verify (kvx_serve.h): argument checks, the workspace, launches.
#include <hip/hip_runtime_api.h>

#include "kvx_host.h"
#include "kvx_verify_internal.h"

namespace {

using kvx::fail;

#define KVX_TRY(call)                              \
    do {                                           \
        const kvx_status status_ = (call);         \
        if (status_ != KVX_OK) return status_;     \
    } while (0)

kvx_status check_drafts(const kvx_drafts* d)
{
    if (!d) return fail(KVX_EINVAL, "NULL drafts");
    if (d->num_requests < 0 || d->total_tokens < 0)
        return fail(KVX_EINVAL, "num_requests and total_tokens must be >= 0");
    if (d->max_tokens < 1 || d->max_tokens > kvx::kMaxDrafted)
        return fail(KVX_EINVAL, "max_tokens %d outside [1, %d]", d->max_tokens, kvx::kMaxDrafted);
    if (d->vocab < 1 || d->vocab > 1 << 24)
        return fail(KVX_EINVAL, "vocab %d outside [1, 2^24]", d->vocab);
    return KVX_OK;
}

int32_t parts_of(const kvx_drafts& d) { return (d.vocab + kvx::kPart - 1) / kvx::kPart; }

// Places `a`'s arrays in a workspace that starts at `base`; returns its size.
uint64_t place(const kvx_drafts& d, bool draft, char* base, kvx::VerifyArgs& a)
{
    uint64_t at = 0;
    auto take = [&](uint64_t bytes) {
        char* const p = base + at;
        at += (bytes + 15) & ~uint64_t(15);
        return p;
    };
    const uint64_t N = d.total_tokens, R = d.num_requests, C = parts_of(d);
    a.part[0] = reinterpret_cast<kvx::Part*>(take(N * C * sizeof(kvx::Part)));
    if (draft) {
        a.part[1] = reinterpret_cast<kvx::Part*>(take(N * C * sizeof(kvx::Part)));
        a.left = reinterpret_cast<double*>(take(N * 8));
        a.residual = reinterpret_cast<double*>(take(R * C * 8));
        a.last = reinterpret_cast<int32_t*>(take(R * 4));
    }
    return at;
}

}  // namespace

extern "C" kvx_status kvx_verify_workspace(const kvx_drafts* d, int32_t with_draft, uint64_t* bytes)
{
    if (!bytes) return fail(KVX_EINVAL, "NULL bytes");
    KVX_TRY(check_drafts(d));
    kvx::VerifyArgs a = {};
    *bytes = d->num_requests == 0 ? 0 : place(*d, with_draft != 0, nullptr, a);
    return KVX_OK;
}

extern "C" kvx_status kvx_verify(const kvx_drafts* d, int32_t dtype, const void* logits, int64_t stride,
                                 const void* draft, int64_t draft_stride, const float* uniforms,
                                 const float* samples, int32_t* accepted, int32_t a_stride,
                                 int32_t* counts, int32_t* next_tokens, void* workspace,
                                 uint64_t workspace_bytes, void* stream)
{
    KVX_TRY(check_drafts(d));
    if (dtype != KVX_FP16 && dtype != KVX_BF16 && dtype != KVX_FP32)
        return fail(KVX_EINVAL, "logits must be KVX_FP16, KVX_BF16 or KVX_FP32, not %d", dtype);
    if (a_stride < 1) return fail(KVX_EINVAL, "a_stride must be >= 1");
    if (d->num_requests == 0) return KVX_OK;
    if (!d->token_starts || !accepted || !counts || !next_tokens)
        return fail(KVX_EINVAL, "NULL token_starts, accepted, counts or next_tokens");
    if (d->total_tokens > 0) {
        if (!d->tokens || !logits || !uniforms || !samples)
            return fail(KVX_EINVAL, "NULL tokens, logits, uniforms or samples");
        if (stride < d->vocab || (draft && draft_stride < d->vocab))
            return fail(KVX_EINVAL, "rows of %d logits at smaller strides", d->vocab);
        const uintptr_t size = dtype == KVX_FP32 ? 4 : 2;
        if (reinterpret_cast<uintptr_t>(logits) % size || reinterpret_cast<uintptr_t>(draft) % size)
            return fail(KVX_EINVAL, "logits must be aligned to their elements");
    }
    kvx::VerifyArgs a = {};
    const uint64_t need = place(*d, draft != nullptr, static_cast<char*>(workspace), a);
    if (need && (!workspace || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 15u)))
        return fail(KVX_EINVAL, "a 16-byte aligned workspace of %llu bytes is needed, %llu are given",
                    (unsigned long long)need, (unsigned long long)(workspace ? workspace_bytes : 0));
    a.starts = d->token_starts;
    a.tokens = d->tokens;
    a.parents = d->parents;
    a.temperatures = d->temperatures;
    a.num_requests = d->num_requests;
    a.total_tokens = d->total_tokens;
    a.max_tokens = d->max_tokens;
    a.vocab = d->vocab;
    a.distinct = d->distinct != 0;
    a.parts = parts_of(*d);
    a.logits = static_cast<const char*>(logits);
    a.draft = static_cast<const char*>(draft);
    a.stride = stride;
    a.draft_stride = draft_stride;
    a.uniforms = uniforms;
    a.samples = samples;
    a.accepted = accepted;
    a.counts = counts;
    a.next = next_tokens;
    a.a_stride = a_stride;
    const double threads = kvx::verify_threads(a);
    if (threads >= 0x1p32) return fail(KVX_EUNSUPPORTED, "%.0f threads in a launch: 2^32 or more", threads);
    int dev = -1;
    const hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return fail(KVX_EDEVICE, "no HIP device: %s", hipGetErrorString(e));
    const int err = kvx::launch_verify(a, dtype, stream);
    if (err != int(hipSuccess))
        return fail(KVX_EDEVICE, "kernel launch failed: %s", hipGetErrorString(hipError_t(err)));
    return KVX_OK;
}
