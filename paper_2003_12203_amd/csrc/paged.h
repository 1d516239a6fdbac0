// Internal definitions of the serving operators: norms and rotation of queries and keys, the paged
// cache of keys and values, and the attention over it.  Not part of the C ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ftcnn_internal.h"

namespace ftcnn {

// Division of a non-negative 32-bit integer by a divisor fixed at the launch.  For d > 1, with
// s = floor(log2(d - 1)) and mul = floor(2^(32 + s) / d) + 1, mul * d exceeds 2^(32 + s) by at most
// d <= 2^(s + 1), so (n * mul) >> (32 + s) is floor(n / d) for every n < 2^31.
struct FastDiv {
    uint32_t d, mul, shift;
};
inline FastDiv fast_div(uint32_t d) {
    FastDiv f{d, 0, 0};
    if (d > 1) {
        while ((2ull << f.shift) <= d - 1) ++f.shift;
        f.mul = (uint32_t)((1ull << (32 + f.shift)) / d + 1);
    }
    return f;
}
__device__ inline uint32_t div_by_many(uint32_t n, const FastDiv &f) { return __umulhi(n, f.mul) >> f.shift; }   // d > 1
__device__ inline uint32_t div_by(uint32_t n, const FastDiv &f) {
    return f.d > 1 ? div_by_many(n, f) : n;
}

struct RopeArgs {
    // sections of a token's heads: 0 queries (or none), 1 keys, 2 values (kv_append)
    const void *x[3];
    void *y[3];
    const void *weight[2];
    long long xs[3][2], ys[3][3];   // elements between tokens and heads; outputs: tokens (or pages, rows) and heads
    int heads[3];
    int chunks[3], all_chunks, per_chunk;   // a lane group takes one token's per_chunk heads of one section
    int tokens, dim, rot, max_pos;
    int interleaved, weight_f32;
    int pages, page;                // kv_append: the cache
    FastDiv div_chunks;
    float eps;
    const int32_t *positions;       // NULL: no rotation
    const int64_t *slots;           // kv_append, else NULL
    const float *table;
};
hipError_t launch_rope_table(const ftcnn_rope_scaling &sc, float *table, hipStream_t st);
hipError_t launch_rope(int dtype, const RopeArgs &a, hipStream_t st);

// A unit that a run of key tiles starts inside of: the first and last run that hold some of it (first_run
// < 0: the run starts with a unit, or is empty), the first row of its sequence's queries, its key head,
// first row of the sequence's rows and count of rows.
struct AttnCut {
    int first_run, last_run, q0, head, r0, rows;
};

struct AttnArgs {
    const void *q, *k, *v;
    void *o;
    float *lse, *part_o, *part_ml;
    AttnCut *cuts;
    const int32_t *page_list, *kv_lens, *q_starts;
    long long qs[2], os[2];      // elements: token, head
    unsigned kb[3], vb[3];       // bytes: page, row, head
    long long list_stride;
    int batch, tokens, kv_heads, group, dim;
    int pages, page, capacity;   // pages of the cache, rows of a page, rows a page list can name
    int causal, window;
    int tiles;                   // whole units: row tiles that the launch has for a sequence
    int groups, min_run;         // even runs (groups > 0): workgroups, and keys that a run has at least
    int unit_cost;               // ... and what the start of a unit counts, in keys
    int tile_keys;
    int part_rows;               // rows of a part in the workspace
    int interleave;              // whole units: pairs of (sequence, key head) dealt to the eight XCDs
    FastDiv div_page, div_group;
    float scale_log2;            // scale * log2(e): the softmax in powers of two
};
// What a call launches.
struct AttnPlan {
    int dp;                      // head size the kernel is compiled for
    int rows, keys;              // of a unit's tiles: 16 rows: stream_kernel, 128: attn_kernel
    int tiles, groups, min_run, unit_cost, part_rows, join_rows;
    size_t part_ml, cuts, bytes;   // workspace: the parts' outputs, their maxima and sums, the cuts
};
AttnPlan attn_plan(const ftcnn_attention_desc &d);
hipError_t launch_attn_bf16(const AttnPlan &pl, const AttnArgs &a, hipStream_t st);
hipError_t launch_attn_f32(const AttnPlan &pl, const AttnArgs &a, hipStream_t st);
hipError_t launch_attn_join(int dtype, const AttnPlan &pl, const AttnArgs &a, hipStream_t st);
hipError_t launch_attn_clear(int dtype, const AttnArgs &a, hipStream_t st);   // a batch of no sequences

// Records the text of ftcnn_last_error() and returns `code`.
int set_error(int code, const char *fmt, ...);

}  // namespace ftcnn
