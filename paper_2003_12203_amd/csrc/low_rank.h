// Internal definitions of the low-rank adapters beside a shared projection.  Not part of the C ABI.
#pragma once

#include "paged.h"

namespace ftcnn {

struct LowRankArgs {
    const void *x, *y, *a, *b;
    void *out;
    const float *scales;          // NULL: 1
    const int32_t *ranks, *ids;   // ranks NULL: all of `rank`
    float *low;                   // [splits][tokens][rank]: s A x of each range of channels
    int4 *records;                // grouped tokens: (adapter, first, how many, 0) of each tile
    int32_t *grouped, *counts;    // the tokens, and how many tiles of each part of them
    long long xs, ys, os;         // elements between tokens
    long long as[2], bs[2];       // elements between adapters, rows
    int tokens, ch, m, adapters, rank;
    int groups, splits;           // groups of rows of A, and ranges of channels, of workgroups of their own
    int ways, expand_ways;        // workgroups that share a tile's adapters, in either launch
    int columns;                  // outputs of a wave of the second launch
    int slots;                    // grouped: records of a part
    FastDiv div_slots;
    FastDiv div_groups, div_splits, div_ways, div_expand_ways, div_spans;
};
struct LowRankPlan {
    bool both;                    // one launch for both products
    bool grouped;                 // tokens are grouped by adapter first
    int parts, slots;             // ... in so many parts, of so many tiles at most
    int tile;                     // tokens of a tile
    int blocks;                   // rows of A of a workgroup, in 16
    int tiles, groups, splits, ways, expand_ways, columns;
    int together, spans;          // tiles of a workgroup of the second launch; its workgroups' spans of outputs
    size_t records, order, count, bytes;   // workspace: after the products
};
LowRankPlan low_rank_plan(const ftcnn_low_rank_desc &d);
hipError_t launch_low_rank(int dtype, const LowRankPlan &pl, const LowRankArgs &a, hipStream_t st);

}  // namespace ftcnn
