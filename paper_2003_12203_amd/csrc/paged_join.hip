// Joins the outputs of the splits of a row's keys: with each split's maximum m_s (in powers of two),
// sum l_s and unnormalised output o_s, O = sum_s 2^(m_s - M) o_s / sum_s 2^(m_s - M) l_s with
// M = max_s m_s, in the order of the splits.  One workgroup a row; its waves' halves take the splits in
// turn, 16 bytes a lane.
#include "paged_attn.h"

namespace ftcnn {
namespace {

template <typename T, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void attn_join_kernel(AttnArgs a, int rows_tile) {
    constexpr int TEAMS = 2 * WAVES;   // 32 lanes each: a split's values, four a lane, in up to two steps
    __shared__ float part[TEAMS][256];
    const int heads = a.kv_heads * a.group;
    const int token = blockIdx.x / heads, head = blockIdx.x % heads;
    const int lane = threadIdx.x & 31, team = threadIdx.x >> 5;
    // the sequence of this token: the last that starts at or before it and is not empty
    int b = token;
    if (a.q_starts) {
        int lo = 0, hi = a.batch;   // starts[lo] <= token < starts[hi], should there be such
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (a.q_starts[mid] <= token) lo = mid;
            else hi = mid;
        }
        b = lo;
    }
    int q0, nq, kv;
    attn_sequence(a, b, q0, nq, kv);
    if (token < q0 || token >= q0 + nq) return;   // nobody's token
    const int first = (token - q0) * a.group + head % a.group;   // its row
    const int r0 = first / rows_tile * rows_tile;
    const int i0 = r0 / a.group, i1 = (min(r0 + rows_tile, nq * a.group) - 1) / a.group;
    int k0, k1;
    const int used = attn_range(a, nq, kv, i0, i1, 0, k0, k1);
    if (used == 1) return;   // the attention kernel wrote it
    const long long orow = blockIdx.x;
    const float *ml = a.part_ml + orow * a.splits * 2, *po = a.part_o + orow * a.splits * a.dim;
    float top = -INFINITY;
    for (int s = threadIdx.x & 63; s < used; s += 64) top = fmaxf(top, ml[2 * s]);
#pragma unroll
    for (int x = 32; x > 0; x /= 2) top = fmaxf(top, __shfl_xor(top, x));
    const float mt = top == -INFINITY ? 0.0f : top;
    float l = 0.0f;
    for (int s = threadIdx.x & 63; s < used; s += 64) l += ml[2 * s + 1] * __builtin_amdgcn_exp2f(ml[2 * s] - mt);
#pragma unroll
    for (int x = 32; x > 0; x /= 2) l += __shfl_xor(l, x);
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    for (int d0 = 0; d0 < a.dim; d0 += 128) {
        const int d = d0 + lane * 4;
        if (d < a.dim) {
            float4 acc = make_float4(0, 0, 0, 0);
#pragma unroll 4
            for (int s = team; s < used; s += TEAMS) {
                const float wgt = __builtin_amdgcn_exp2f(ml[2 * s] - mt);
                const float4 v = *reinterpret_cast<const float4 *>(po + (long long)s * a.dim + d);
                acc.x = fmaf(wgt, v.x, acc.x);
                acc.y = fmaf(wgt, v.y, acc.y);
                acc.z = fmaf(wgt, v.z, acc.z);
                acc.w = fmaf(wgt, v.w, acc.w);
            }
            *reinterpret_cast<float4 *>(&part[team][d]) = acc;
        }
    }
    __syncthreads();
    T *out = static_cast<T *>(a.o) + (long long)token * a.os[0] + (long long)head * a.os[1];
    for (int d = threadIdx.x; d < a.dim; d += 64 * WAVES) {
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < TEAMS; ++k) sum += part[k][d];
        Elem<T>::store(out, d, sum * inv);
    }
    if (a.lse && threadIdx.x == 0) a.lse[orow] = l == 0.0f ? -INFINITY : (mt + __log2f(l)) * 0.693147180559945309f;
}

template <typename T> hipError_t go(const AttnPlan &pl, const AttnArgs &a, hipStream_t st) {
    const unsigned rows = (unsigned)(a.tokens * a.kv_heads * a.group);
    if (a.splits <= 8) attn_join_kernel<T, 1><<<rows, 64, 0, st>>>(a, pl.wr * 32);
    else attn_join_kernel<T, 4><<<rows, 256, 0, st>>>(a, pl.wr * 32);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_attn_join(int dtype, const AttnPlan &pl, const AttnArgs &a, hipStream_t st) {
    return dtype == FTCNN_F32 ? go<float>(pl, a, st) : go<uint16_t>(pl, a, st);
}

}  // namespace ftcnn
