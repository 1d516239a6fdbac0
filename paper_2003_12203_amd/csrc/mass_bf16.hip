// bf16 instances of the attention weights' kernels, their plan, and the sum of the parts.
#include "mass_kernel.h"

namespace ftcnn {
namespace {

constexpr int kJoinKeys = 32, kJoinShares = kThreads / kJoinKeys;   // of a workgroup; lanes that share a key's parts

// mass += the parts, the shares' sums and theirs in an order that the count of parts alone decides.
__global__ __launch_bounds__(kThreads) void mass_join_kernel(MassArgs p, int parts) {
    __shared__ float sums[kJoinShares][kJoinKeys];
    const int b = (int)(blockIdx.x % (unsigned)p.t.batch), step = (int)(gridDim.x / (unsigned)p.t.batch);
    const int n = min(max(p.t.kv_lens[b], 0), p.t.capacity), blocks = (n + kJoinKeys - 1) / kJoinKeys;
    const int in = threadIdx.x % kJoinKeys, share = threadIdx.x / kJoinKeys;
    const long long each = (long long)p.t.batch * p.t.capacity;
    for (int block = (int)(blockIdx.x / (unsigned)p.t.batch); block < blocks; block += step) {
        const int j = block * kJoinKeys + in;
        float v = 0.0f;
        if (j < n) {
            const float *part = p.part + (long long)b * p.t.capacity + j;
#pragma unroll 4
            for (int i = share; i < parts; i += kJoinShares) v += part[i * each];
        }
        __syncthreads();   // the block before this one
        sums[share][in] = v;
        __syncthreads();
        if (share == 0 && j < n) {
#pragma unroll
            for (int i = 1; i < kJoinShares; ++i) v += sums[i][in];
            p.mass[b * p.mass_stride + j] += v;
        }
    }
}

}  // namespace

hipError_t launch_mass_bf16(const MassPlan &pl, const MassArgs &a, hipStream_t st) { return mass_pick<uint16_t>(pl, a, st); }

hipError_t launch_mass_join(const MassPlan &pl, const MassArgs &a, hipStream_t st) {
    const long long blocks = std::max(1LL, std::min(((long long)pl.blocks * pl.keys + kJoinKeys - 1) / kJoinKeys,
                                                    8192LL / a.t.batch));
    mass_join_kernel<<<(unsigned)(blocks * a.t.batch), kThreads, 0, st>>>(a, pl.head_parts * pl.row_parts);
    return hipGetLastError();
}

}  // namespace ftcnn
