// bf16 instances of the attention weights' kernels, their plan, and the sum of the parts.
#include "mass_kernel.h"

namespace ftcnn {
namespace {

// mass += the parts, in their order.
__global__ __launch_bounds__(kThreads) void mass_join_kernel(MassArgs p, int parts) {
    const int b = (int)(blockIdx.x % (unsigned)p.t.batch);
    const int n = min(max(p.t.kv_lens[b], 0), p.t.capacity);
    const long long step = (long long)p.t.batch * p.t.capacity;
    float *mass = p.mass + b * p.mass_stride;
    const int each = (int)(gridDim.x / (unsigned)p.t.batch) * kThreads;
    for (long long j = (int)(blockIdx.x / (unsigned)p.t.batch) * kThreads + threadIdx.x; j < n; j += each) {
        const float *part = p.part + (long long)b * p.t.capacity + j;
        float v = 0.0f;
        for (int i = 0; i < parts; ++i) v += part[i * step];
        mass[j] += v;
    }
}

}  // namespace

hipError_t launch_mass_bf16(const MassPlan &pl, const MassArgs &a, hipStream_t st) { return mass_pick<uint16_t>(pl, a, st); }

hipError_t launch_mass_join(const MassPlan &pl, const MassArgs &a, hipStream_t st) {
    const long long blocks = std::max(1LL, std::min(((long long)pl.blocks * pl.keys + kThreads - 1) / kThreads,
                                                    4096LL / a.t.batch));
    mass_join_kernel<<<(unsigned)(blocks * a.t.batch), kThreads, 0, st>>>(a, pl.head_parts * pl.row_parts);
    return hipGetLastError();
}

}  // namespace ftcnn
