// bf16 instances of the attention kernel.
#include "paged_stream.h"

namespace ftcnn {
namespace {
template <int DP> hipError_t pick(const AttnPlan &pl, const AttnArgs &a, hipStream_t st) {
    if (pl.rows == 16) return stream_go<uint16_t, DP>(a, st);
    return attn_go<uint16_t, DP, 4, (DP <= 128 ? 2 : 1)>(a, st);
}
}  // namespace

hipError_t launch_attn_bf16(const AttnPlan &pl, const AttnArgs &a, hipStream_t st) {
    if (pl.dp == 64) return pick<64>(pl, a, st);
    if (pl.dp == 128) return pick<128>(pl, a, st);
    return pick<256>(pl, a, st);
}

}  // namespace ftcnn
