// Internal definitions of the eviction from a paged cache.  Not part of the C ABI.
#pragma once

#include "paged.h"

namespace ftcnn {

constexpr int kEvictHeld = 16384;   // places that a workgroup keeps, at most
// Longer sequences are chosen from in parts of so many places, and a part finds for the others:
constexpr int kEvictPart = 8192, kEvictBins = 2048, kEvictWaves = 16;
struct alignas(16) EvictPart {
    uint32_t bins[4][kEvictBins];   // counts of bits: of the first pass, the second, the third; the first of those kept for their positions
    uint4 found[3];                 // of the first part: the limit after each pass
    uint32_t kept, holes, late;     // kept for their positions; moves' places below k and rows from k on
    uint32_t hole_at[kEvictWaves], late_at[kEvictWaves], rank[kEvictWaves];   // of the waves, in the part; of ties in all
};

struct EvictArgs {
    void *k, *v;
    unsigned kb[3], vb[3];        // bytes: page, row, head
    const int32_t *page_list, *kv_lens, *keep, *positions, *since;
    const float *mass;
    int32_t *lens_out, *positions_out;
    float *mass_out;
    long long list_stride, ms, ps, mos, pos;   // elements between sequences: mass, positions, and those written
    int batch, kv_heads, pages, page, capacity, first;
    int units;                    // 16-byte units of a row of a head
    int32_t *counts, *from, *to;  // workspace: moves of each sequence, [batch] and [batch][half]
    long long half;
    int parts;                    // of a sequence, or 0: a workgroup's each
    EvictPart *part;              // workspace [batch][parts]
    int held;                     // places of a workgroup whose weights and positions it keeps in LDS
    int shares;                   // workgroups that share a sequence's moves
    FastDiv div_page;
};
hipError_t launch_evict(const EvictArgs &a, hipStream_t st);

}  // namespace ftcnn
