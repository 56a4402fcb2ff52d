// Internal declarations shared by the host side of the decode operators
// (kvx_ops.cpp) and their kernels: kvx_slots.hip (append, evict, commit),
// kvx_attend.hip with kvx_attend_few.hip and kvx_attend_rows*, kvx_weigh.hip.
#pragma once

#include <cstdint>

#include "kvx_internal.h"
#include "kvx_ops.h"

namespace kvx {

// One layer range of a cache as the kernels address it.  A plane is the pages
// of one (layer, k/v): [num_blocks][block_size][hd][dim].
struct CacheArgs {
    char* base;                  // plane (layer0, k)
    float* scales;               // its scales, NULL for 16-bit elements
    const int32_t* table;
    int64_t plane_bytes;         // bytes between planes
    int64_t plane_scales;        // scales between planes
    int64_t num_blocks;
    int32_t bt_stride;
    int32_t block_size;
    int32_t hd;
    int32_t dim;
    int32_t row_bytes;           // dim x element size
    int32_t row_slots;           // slots of a block-table row: bt_stride x block_size, cut to int32
    int32_t num_requests;
    int32_t pad;
    FastDiv div_bs;              // by block_size
};

struct BatchArgs {
    const int32_t* starts;
    const int32_t* contexts;
    const int32_t* positions;
    const uint64_t* tree;
    int32_t tree_stride;
    int32_t total_tokens;
    int32_t max_tokens;
    int32_t max_context;
};

struct AppendArgs {
    CacheArgs c;
    BatchArgs b;
    const uint16_t* q;
    const uint16_t* k;
    const uint16_t* v;
    uint16_t* q_out;
    int64_t q_stride, k_stride, v_stride, q_out_stride;
    const float* inv_freq;
    const int32_t* positions;    // [axes][N]
    int32_t q_heads;
    int32_t pairs;
    int32_t interleaved;
    int32_t sec_end[4];          // pairs below sec_end[a] belong to an axis <= a
    int32_t lg_row;              // log2 of the lanes per head: a power of two >= dim / 8
};

struct EvictArgs {
    CacheArgs c;
    const int32_t* lens;
    const float* weights;
    float* weights_out;
    int32_t* kept;
    int32_t* new_lens;
    int64_t w_stride;
    int32_t max_len, budget, sink, recent;
};

// What an eviction moves: in every plane and head, row i of request r takes row
// kept[i], for `budget` rows where lens[r] is above that, else none.
struct MoveArgs {
    CacheArgs c;
    const int32_t* kept;         // [layer][request][head][budget], ascending
    const int32_t* lens;
    int32_t budget;
    int32_t max_len;
    int32_t lg_lanes;            // log2 of the lanes that a head's row takes
    int32_t pad;
};

// In every plane, row contexts[r] + i of request r takes row contexts[r] +
// accepted[i], all heads, for a path of counts[r] entries or fewer, whose end goes
// to new_lens[r].
struct CommitArgs {
    CacheArgs c;
    const int32_t* contexts;
    const int32_t* accepted;     // [request][a_stride], ascending
    const int32_t* counts;
    int32_t* new_lens;
    int32_t a_stride;
    int32_t num_layers;
    int32_t lg_lanes;            // log2 of the lanes that all heads' rows take
    int32_t pad;
};

struct AttendArgs {
    CacheArgs c;                 // base: the layer's k plane
    BatchArgs b;
    const uint16_t* q;
    uint16_t* out;
    float* lse;                  // weigh: read
    float* weights;              // weigh
    int64_t q_stride, out_stride, w_stride;
    const float* slopes;
    const int32_t* prefix;
    float scale, softcap;
    int32_t window;
    int32_t q_heads;
    int32_t group;
    FastDiv div_group;
    // a request's slots are dealt to `splits` workgroups, `chunk` slots each; more than one
    // leave their sums here for kvx_join_kernel: part_o [split][N][q_heads][dim] and
    // part_ml [split][N][q_heads] pairs (reference, sum of weights)
    int32_t chunk, splits;
    float* part_o;
    float* part_ml;
};

// How a call is cut into workgroups.
struct AttendPlan {
    int rows;            // query rows of a KV head, at most
    bool few;            // kvx_attend_few_kernel, else kvx_attend_rows_kernel
    int row_tiles;       // workgroups along the rows (1 for few)
    int tile_rows;       // rows of a workgroup
    int chunk, splits;
};
AttendPlan attend_plan(const kvx_cache& c, const kvx_batch& b, int32_t q_heads);
int launch_few(const AttendArgs& a, const AttendPlan& p, int dtype, int cache_dtype, void* stream);
template <int kCodes>
int launch_rows(const AttendArgs& a, const AttendPlan& p, int dtype, void* stream);

// The threads of a call's largest launch, workgroups times their size: HIP takes
// fewer than 2^32.
double append_threads(int32_t tokens);
double evict_threads(const CacheArgs& c, int num_layers, int max_len);
double commit_threads(const CacheArgs& c, int num_layers);
double attend_threads(const kvx_cache& c, const kvx_batch& b, int32_t q_heads, const AttendPlan& p);
double weigh_threads(const kvx_cache& c, const kvx_batch& b, int32_t q_heads);

// Each enqueues its kernels on `stream` and returns a hipError_t value.
int launch_append(const AppendArgs& a, int dtype, int cache_dtype, void* stream);
int launch_evict(const EvictArgs& a, int num_layers, void* stream);
int launch_commit(const CommitArgs& a, void* stream);
int launch_attend(const AttendArgs& a, const AttendPlan& p, int dtype, int cache_dtype,
                  void* workspace, void* stream);
int launch_weigh(const AttendArgs& a, int dtype, int cache_dtype, void* stream);
uint64_t attend_workspace(const kvx_cache& c, const kvx_batch& b, int32_t q_heads);

}  // namespace kvx
