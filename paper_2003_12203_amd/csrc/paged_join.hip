// Joins the parts of a unit whose keys several workgroups walked: with each part's maximum m_s (in powers
// of two), sum l_s and unnormalised output o_s of a row,
//   O = sum_s 2^(m_s - M) o_s / sum_s 2^(m_s - M) l_s,  M = max_s m_s,
// in an order that the parts' count and place alone decide.  The run that a unit's second part lies in says
// what there is to join (AttnCut).  A workgroup looks through some of the runs and takes some of each such
// unit's rows: a team of 32 lanes (four values a lane) a row, or with fewer rows than teams several that
// share a row's parts.
//
// It reads each part once: chunks over 8192 cached tokens, 64 MB of parts, 18 to 20 us; single tokens of 64 sequences 6 to 7 us
// (2048, 4096 or 8192 workgroups, or parts loaded before their weights are known: the same).
#include <algorithm>

#include "paged_attn.h"

namespace ftcnn {
namespace {

constexpr int kTeams = kThreads / 32;
constexpr int kInFlight = 8;   // parts that a team has on their way

template <typename T>
__global__ __launch_bounds__(kThreads) void attn_join_kernel(AttnArgs a, int rows_here) {
    __shared__ float4 sums[kTeams][64];
    const int lane = threadIdx.x & 31, team = threadIdx.x >> 5;
    const int wave_lane = threadIdx.x & 63;
    for (int c0 = blockIdx.x; c0 < a.groups; c0 += 64 * gridDim.x) {
        // the runs of this workgroup that a unit's second part lies in
        const long long mine = c0 + (long long)wave_lane * gridDim.x;
        unsigned long long owned = __ballot(mine < a.groups && a.cuts[min(mine, a.groups - 1LL)].first_run == mine - 1 &&
                                            mine > 0);
        for (; owned; owned &= owned - 1) {
            const AttnCut cut = a.cuts[c0 + __builtin_ctzll(owned) * gridDim.x];
            const int from = blockIdx.y * rows_here, rows = min(cut.rows - from, rows_here);
            if (rows <= 0) continue;
            const int parts = cut.last_run - cut.first_run + 1;
            const int share = rows > 4 ? 1 : (rows > 2 ? 2 : (rows > 1 ? 4 : 8));   // teams a row
            const int sub = team % share;
            for (int r0 = 0; r0 < rows; r0 += kTeams / share) {
                const int row = from + r0 + team / share;
                const bool ok = row < from + rows;
                auto at = [&](int s) { return attn_part(cut.first_run + s, s == 0) * a.part_rows + row; };
                float l = 0.0f, mt = 0.0f;
                float4 acc[2] = {make_float4(0, 0, 0, 0), make_float4(0, 0, 0, 0)};
                if (ok) {
                    // maximum and sum of up to 256 parts at a time, all their loads in flight
                    float top = -INFINITY;
                    for (int s0 = lane; s0 < parts; s0 += 256) {
                        float2 r[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k)
                            r[k] = s0 + 32 * k < parts ? *reinterpret_cast<const float2 *>(a.part_ml + 2 * at(s0 + 32 * k))
                                                       : make_float2(-INFINITY, 0.0f);
                        float t = top;
#pragma unroll
                        for (int k = 0; k < 8; ++k) t = fmaxf(t, r[k].x);
                        const float t0 = t == -INFINITY ? 0.0f : t;
                        l *= __builtin_amdgcn_exp2f(top - t0);
#pragma unroll
                        for (int k = 0; k < 8; ++k) l += r[k].y * __builtin_amdgcn_exp2f(r[k].x - t0);
                        top = t;
                    }
                    float all = top;
#pragma unroll
                    for (int x = 16; x > 0; x /= 2) all = fmaxf(all, __shfl_xor(all, x, 32));
                    mt = all == -INFINITY ? 0.0f : all;
                    l *= __builtin_amdgcn_exp2f(top - mt);
#pragma unroll
                    for (int x = 16; x > 0; x /= 2) l += __shfl_xor(l, x, 32);
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const int d = k * 128 + lane * 4;
                        if (d >= a.dim) continue;
                        for (int s0 = sub; s0 < parts; s0 += kInFlight * share) {
                            float at_max[kInFlight];
                            float4 v[kInFlight];
#pragma unroll
                            for (int x = 0; x < kInFlight; ++x) {
                                const long long p = at(min(s0 + x * share, parts - 1));
                                at_max[x] = a.part_ml[2 * p];
                                v[x] = *reinterpret_cast<const float4 *>(a.part_o + p * a.dim + d);
                            }
#pragma unroll
                            for (int x = 0; x < kInFlight; ++x) {
                                // (no branch: it would have each load wait for the one before)
                                const bool there = s0 + x * share < parts;
                                const float wgt = there ? __builtin_amdgcn_exp2f(at_max[x] - mt) : 0.0f;
                                acc[k].x = fmaf(wgt, there ? v[x].x : 0.0f, acc[k].x);
                                acc[k].y = fmaf(wgt, there ? v[x].y : 0.0f, acc[k].y);
                                acc[k].z = fmaf(wgt, there ? v[x].z : 0.0f, acc[k].z);
                                acc[k].w = fmaf(wgt, there ? v[x].w : 0.0f, acc[k].w);
                            }
                        }
                    }
                }
                if (share > 1) {   // a workgroup's threads agree on it
                    __syncthreads();
                    sums[team][lane] = acc[0];
                    sums[team][32 + lane] = acc[1];
                    __syncthreads();
                    if (sub == 0)
                        for (int k = 1; k < share; ++k)
#pragma unroll
                            for (int x = 0; x < 2; ++x) {
                                const float4 v = sums[team + k][32 * x + lane];
                                acc[x].x += v.x;
                                acc[x].y += v.y;
                                acc[x].z += v.z;
                                acc[x].w += v.w;
                            }
                }
                if (!ok || sub) continue;
                const float inv = l == 0.0f ? 0.0f : 1.0f / l;
                const int i = (int)div_by(cut.r0 + row, a.div_group);
                const int head = cut.head * a.group + cut.r0 + row - i * a.group;
                T *out = static_cast<T *>(a.o) + (long long)(cut.q0 + i) * a.os[0] + (long long)head * a.os[1];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int d = k * 128 + lane * 4;
                    if (d < a.dim)
                        store4(out + d, make_float4(acc[k].x * inv, acc[k].y * inv, acc[k].z * inv, acc[k].w * inv));
                }
                if (a.lse && lane == 0)
                    a.lse[(long long)(cut.q0 + i) * a.kv_heads * a.group + head] =
                        l == 0.0f ? -INFINITY : (mt + __log2f(l)) * 0.693147180559945309f;
            }
        }
    }
}

template <typename T> __global__ __launch_bounds__(kThreads) void attn_clear_kernel(AttnArgs a) {
    attn_clear_unowned<T, kThreads>(a);
}

}  // namespace

hipError_t launch_attn_clear(int dtype, const AttnArgs &a, hipStream_t st) {
    const unsigned blocks = (unsigned)std::min(a.tokens, 2048);
    if (dtype == FTCNN_F32) attn_clear_kernel<float><<<blocks, kThreads, 0, st>>>(a);
    else attn_clear_kernel<uint16_t><<<blocks, kThreads, 0, st>>>(a);
    return hipGetLastError();
}

hipError_t launch_attn_join(int dtype, const AttnPlan &pl, const AttnArgs &a, hipStream_t st) {
    // rows of a unit to a workgroup, and workgroups to look through the runs: about 2048 in all
    const int y = (pl.part_rows + pl.join_rows - 1) / pl.join_rows;
    const dim3 grid((unsigned)std::min(pl.groups, std::max(64, 2048 / y)), (unsigned)y);
    if (dtype == FTCNN_F32) attn_join_kernel<float><<<grid, kThreads, 0, st>>>(a, pl.join_rows);
    else attn_join_kernel<uint16_t><<<grid, kThreads, 0, st>>>(a, pl.join_rows);
    return hipGetLastError();
}

}  // namespace ftcnn
