// Internal definitions of the low-rank adapters beside a shared projection.  Not part of the C ABI.
#pragma once

#include "paged.h"

namespace ftcnn {

struct LowRankArgs {
    const void *x, *y, *a, *b;
    void *out;
    const float *scales;          // NULL: 1
    const int32_t *ranks, *ids;   // ranks NULL: all of `rank`
    float *part;                  // [splits][tokens][rank]: s A x of each range of channels
    long long xs, ys, os;         // elements between tokens
    long long as[2], bs[2];       // elements between adapters, rows
    int tokens, ch, m, adapters, rank;
    int splits;                   // ranges of channels
    int tiles, ways;              // tiles of tokens; workgroups that share a tile's adapters, in either launch
    int expand_ways, columns;     // outputs of a workgroup of the second launch
};
struct LowRankPlan {
    int tile;                     // tokens of a tile
    int splits, tiles, ways, expand_ways, columns;
    size_t bytes;
};
LowRankPlan low_rank_plan(const ftcnn_low_rank_desc &d);
hipError_t launch_low_rank(int dtype, const LowRankPlan &pl, const LowRankArgs &a, hipStream_t st);

}  // namespace ftcnn
