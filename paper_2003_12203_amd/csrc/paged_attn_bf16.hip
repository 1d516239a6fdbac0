// bf16 instances of the attention kernel.
#include "paged_attn.h"

namespace ftcnn {
namespace {
template <int DP> hipError_t pick(const AttnPlan &pl, const AttnArgs &a, hipStream_t st) {
    constexpr bool wide = DP > 128;
    if (pl.wr == 1) return attn_go<uint16_t, DP, 1, wide ? 2 : 4, 1>(a, st);
    if (pl.wr == 2) return attn_go<uint16_t, DP, 2, 2, 1>(a, st);
    return attn_go<uint16_t, DP, wide ? 4 : 8, 1, wide ? 1 : 2>(a, st);
}
}  // namespace

hipError_t launch_attn_bf16(const AttnPlan &pl, const AttnArgs &a, hipStream_t st) {
    if (pl.dp == 64) return pick<64>(pl, a, st);
    if (pl.dp == 128) return pick<128>(pl, a, st);
    return pick<256>(pl, a, st);
}

}  // namespace ftcnn
