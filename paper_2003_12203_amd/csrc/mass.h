// Internal definitions of the accumulated attention weights.  Not part of the C ABI.
#pragma once

#include "paged.h"

namespace ftcnn {

struct MassArgs {
    AttnArgs t;                  // queries, keys, page lists, lengths, the mask; no values, outputs or schedule
    const float *lse;            // [tokens][heads]
    float *mass, *part;          // part [parts][batch][capacity], where parts > 1
    long long mass_stride;
    int blocks;                  // blocks of keys that the launch has for a sequence
    int head_parts, row_parts;   // workgroups that share a block's key heads, and its rows
    FastDiv div_heads, div_rows, div_blocks;   // by head_parts, row_parts, blocks
    bool near;                   // 64 rows of the queries lie within 2^32 bytes
};
struct MassPlan {
    int dp;                      // head size the kernel is compiled for
    bool wide;                   // more than 64 rows of a key head
    int keys;                    // of a workgroup
    int blocks, head_parts, row_parts;
    size_t bytes;
};
MassPlan mass_plan(const ftcnn_mass_desc &d);
hipError_t launch_mass_bf16(const MassPlan &pl, const MassArgs &a, hipStream_t st);
hipError_t launch_mass_f32(const MassPlan &pl, const MassArgs &a, hipStream_t st);
hipError_t launch_mass_join(const MassPlan &pl, const MassArgs &a, hipStream_t st);

}  // namespace ftcnn
