// What the host side of kvx_verify (kvx_verify.cpp) and its kernels
// (kvx_verify.hip) share.
#pragma once

#include <cstdint>

#include "kvx_serve.h"

namespace kvx {

constexpr int32_t kMaxDrafted = 1024;    // tokens of a request
constexpr int32_t kPart = 4096;          // logits of a part of a row

// A part of a row: its largest logit, where that first is, and the sum of exp((l - top) / T);
// NaN where one of them is NaN or +infinity.
struct Part {
    double sum;
    float top;
    int32_t at;
};

struct VerifyArgs {
    const int32_t* starts;
    const int32_t* tokens;
    const int32_t* parents;
    const float* temperatures;
    int32_t num_requests, total_tokens, max_tokens, vocab;
    int32_t distinct, parts;             // parts of a row
    const char* logits;
    const char* draft;                   // NULL: none
    int64_t stride, draft_stride;        // elements
    const float* uniforms;
    const float* samples;
    int32_t* accepted;
    int32_t* counts;
    int32_t* next;
    int32_t a_stride, pad;
    // workspace
    Part* part[2];                       // [N][parts] of the target's and the draft's rows
    double* left;                        // [N]: 1 / sum of what a token's refusal leaves of r
    double* residual;                    // [R][parts]: sums of r after the last token
    int32_t* last;                       // [R]: it (kLeaf: a leaf), -1: none; with a draft
};

// Enqueues the kernels of a call; returns a hipError_t value.
int launch_verify(const VerifyArgs& a, int dtype, void* stream);
// The threads of its largest launch.
double verify_threads(const VerifyArgs& a);

}  // namespace kvx
