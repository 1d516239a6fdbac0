// Attention of new tokens over a paged cache of keys and values: the kernel.
//
//   S_ij = scale * q_i . k_j over the keys j that row i sees,
//   O_i = sum_j exp(S_ij - m_i) v_j / l_i,  l_i = sum_j exp(S_ij - m_i),  m_i = max_j S_ij,
//
// in one pass over the keys with the running maximum m and sum l, all of these in fp32 (powers of
// two: exp(x) = 2^(x log2 e)).  Rows are (new token, query head of one key head) pairs, so all the
// queries that share a key head share its loads; a workgroup owns WR x 32 rows and walks the keys in
// tiles of 32 KS WK, which 16-byte loads move straight into LDS, one tile ahead.
//
// The products run transposed.  S^T = K Q^T has a row's scores in one lane and its other half
// (lane ^ 32): softmax needs one exchange.  A lane then holds the keys 8 q + 4 half + (0..3), and
// O^T = V^T P^T takes any order of its keys as long as both operands have the same: P stays in
// registers, rounded to bf16 (fp32 kernels: as it is), and V is read from LDS in that order (bf16:
// transposed on the way, four keys of 16 columns at a time).
//
// LDS rows are unpadded (the direct loads write 1024 consecutive bytes a wave); 16-byte units are
// permuted within a row instead, so that what a cycle reads falls on different banks: the loads fetch
// the unit that belongs at their place.
#pragma once

#include "paged.h"

namespace ftcnn {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) void attn_lds_t;
typedef __attribute__((address_space(1))) const void attn_global_t;

// Zeros for the columns past the head's size, which the loads of a wider kernel fetch.
__device__ __align__(16) const uint32_t attn_zero[4] = {0, 0, 0, 0};

// The keys [k0, k1) of split `split` of the rows of tokens i0..i1 of a sequence with nq new and kv
// cached tokens; returns the splits these rows use (at least one).
__device__ inline int attn_range(const AttnArgs &a, int nq, int kv, int i0, int i1, int split, int &k0, int &k1) {
    const int past = kv - nq;
    int hi = kv, lo = 0;
    if (a.causal) hi = min(kv, max(0, past + i1 + 1));
    if (a.window > 0) lo = min(hi, max(0, past + i0 - a.window + 1));
    const int n = min(a.splits, max(1, (hi - lo + a.per_split - 1) / a.per_split));
    k0 = lo + split * a.per_split;
    k1 = split == n - 1 ? hi : k0 + a.per_split;
    return n;
}

// A sequence's new tokens [q0, q0 + nq) and cached tokens, within what the caller's arrays hold.
__device__ inline void attn_sequence(const AttnArgs &a, int b, int &q0, int &nq, int &kv) {
    if (a.q_starts) {
        q0 = min(max(a.q_starts[b], 0), a.tokens);
        nq = min(max(a.q_starts[b + 1], q0), a.tokens) - q0;
    } else {
        q0 = b;
        nq = 1;
    }
    kv = min(max(a.kv_lens[b], 0), a.capacity);
}

template <typename T, int DP, int WR, int WK, int KS> struct AttnTile {
    static constexpr int NW = WR * WK, THREADS = 64 * NW, ROWS = 32 * WR, KEYS = 32 * KS * WK;
    static constexpr int EU = 16 / sizeof(T);          // values of a 16-byte unit
    static constexpr int UPR = DP / EU;                // units of a row
    static constexpr int RB = DP * (int)sizeof(T);     // bytes of a row
    static constexpr int SIDE = KEYS * RB;             // bytes of a tile of keys, or of values
    static constexpr int LOADS = KEYS * UPR / THREADS;
    static constexpr int JOIN = WK > 1 ? NW * 32 * DP * 4 + NW * 256 : 0;
    static constexpr int LDS = 4 * SIDE > JOIN ? 4 * SIDE : JOIN;
    static_assert(KEYS * UPR % THREADS == 0 && 64 % UPR == 0, "whole loads");
    // where unit u of row r lies.  Keys: 16 lanes read the same unit of 16 consecutive rows.
    __device__ static int key_unit(int r) { return UPR == 8 ? (r >> 1) & 7 : r & 15; }
    // Values: 32 lanes read 64 bytes of four consecutive rows (bf16), or 128 bytes of rows r and r + 4.
    __device__ static int value_unit(int r) {
        if (sizeof(T) == 4) return ((r >> 2) & 1) << 3;
        return UPR == 8 ? ((r >> 1) & 1) << 2 : (r & 3) << 2;
    }
};

template <typename T, int DP, int WR, int WK, int KS>
__global__ __launch_bounds__(64 * WR * WK) void attn_kernel(AttnArgs a) {
    using L = AttnTile<T, DP, WR, WK, KS>;
    constexpr bool BF = sizeof(T) == 2;
    constexpr int UPR = L::UPR, EU = L::EU, RB = L::RB, NQ = UPR / 2, ND = DP / 32;
    extern __shared__ __align__(1024) unsigned char lds[];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, half = lane >> 5, wr = w / WK, wk = w % WK;

    // workgroup -> (sequence b, key head, split, tile of rows); the last tiles, with the most keys, first
    unsigned id = blockIdx.x;
    const unsigned per_pair = (unsigned)a.tiles * a.splits;
    unsigned pair, in;
    if (a.interleave) {   // a pair's workgroups on one XCD, whose L2 then holds its keys and values
        const unsigned s = id >> 3;
        pair = (s / per_pair) * 8 + (id & 7);
        in = s % per_pair;
    } else {
        pair = id / per_pair;
        in = id % per_pair;
    }
    const int hk = (int)(pair % (unsigned)a.kv_heads), b = (int)(pair / (unsigned)a.kv_heads);
    const int split = (int)(in / (unsigned)a.tiles), tile0 = a.tiles - 1 - (int)(in % (unsigned)a.tiles);
    int q0, nq, kv;
    attn_sequence(a, b, q0, nq, kv);
    const int rows = nq * a.group;
    const T *kbase = static_cast<const T *>(a.k) + (long long)hk * a.ks[2];
    const T *vbase = static_cast<const T *>(a.v) + (long long)hk * a.vs[2];
    const int32_t *list = a.page_list + (long long)b * a.list_stride;
    const float c = a.scale_log2;

    // a lane's part of the loads: load i fills its unit of row row0 + i * STEP
    constexpr int STEP = L::THREADS / UPR;
    const int row0 = tid / UPR, slot = tid % UPR;

    for (int tile = tile0; tile * L::ROWS < rows; tile += a.tiles) {
        const int r0 = tile * L::ROWS;
        const int i0 = (int)div_by(r0, a.div_group), i1 = (int)div_by(min(r0 + L::ROWS, rows) - 1, a.div_group);
        int k0, k1;
        const int used = attn_range(a, nq, kv, i0, i1, split, k0, k1);
        if (split >= used) continue;

        // this lane's row; past the last one, the last again (not stored)
        const int r = min(r0 + wr * 32 + l32, rows - 1);
        const bool stored = r0 + wr * 32 + l32 < rows, idle = r0 + wr * 32 >= rows;
        const int qi = (int)div_by(r, a.div_group), head = hk * a.group + r - qi * a.group;
        const int pos = kv - nq + qi;
        const int jhi = min(a.causal ? pos : kv - 1, k1 - 1);      // the keys it sees: jlo..jhi
        const int jlo = a.window > 0 ? pos - a.window + 1 : 0;
        const int jhi_min = __builtin_amdgcn_readlane(jhi, 0), jhi_max = __builtin_amdgcn_readlane(jhi, 31);
        const int jlo_min = __builtin_amdgcn_readlane(jlo, 0), jlo_max = __builtin_amdgcn_readlane(jlo, 31);

        // queries: unit 2 t + half of the row
        uint4 qf[NQ];
        {
            const T *qrow = static_cast<const T *>(a.q) + (long long)(q0 + qi) * a.qs[0] + (long long)head * a.qs[1];
#pragma unroll
            for (int t = 0; t < NQ; ++t) {
                const int u = 2 * t + half;
                qf[t] = u * EU < a.dim ? *reinterpret_cast<const uint4 *>(qrow + u * EU) : make_uint4(0, 0, 0, 0);
            }
        }
        f32x16 o[ND];
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[d][e] = 0.0f;
        float m = -INFINITY, l = 0.0f;

        int pid[L::LOADS];
        auto key_of = [&](int t, int i) { return min(k0 + t * L::KEYS + row0 + i * STEP, k1 - 1); };
        auto lookup = [&](int t) {
#pragma unroll
            for (int i = 0; i < L::LOADS; ++i)
                pid[i] = min(max(list[div_by(key_of(t, i), a.div_page)], 0), a.pages - 1);
        };
        auto issue = [&](int t, int buf) {
#pragma unroll
            for (int i = 0; i < L::LOADS; ++i) {
                const int key = key_of(t, i), in_page = key - (int)div_by(key, a.div_page) * a.page;
                const int row = row0 + i * STEP;
                unsigned char *to = lds + buf * 2 * L::SIDE + (i * L::THREADS + w * 64) * 16;
                const int uk = slot ^ L::key_unit(row), uv = slot ^ L::value_unit(row);
                const T *pk = kbase + (long long)pid[i] * a.ks[0] + (long long)in_page * a.ks[1] + uk * EU;
                const T *pv = vbase + (long long)pid[i] * a.vs[0] + (long long)in_page * a.vs[1] + uv * EU;
                if (DP != a.dim) {
                    if (uk * EU >= a.dim) pk = reinterpret_cast<const T *>(attn_zero);
                    if (uv * EU >= a.dim) pv = reinterpret_cast<const T *>(attn_zero);
                }
                __builtin_amdgcn_global_load_lds((attn_global_t *)pk, (attn_lds_t *)to, 16, 0, 0);
                __builtin_amdgcn_global_load_lds((attn_global_t *)pv, (attn_lds_t *)(to + L::SIDE), 16, 0, 0);
            }
        };

        const int ntiles = (k1 - k0 + L::KEYS - 1) / L::KEYS;
        __syncthreads();   // the tile of rows before this one may still read LDS
        if (ntiles > 0) {
            lookup(0);
            issue(0, 0);
            if (ntiles > 1) lookup(1);
        }
        for (int t = 0; t < ntiles; ++t) {
            __syncthreads();   // this tile has landed, and nobody reads the other buffer any more
            if (t + 1 < ntiles) issue(t + 1, (t + 1) & 1);
            if (t + 2 < ntiles) lookup(t + 2);
            const unsigned char *kt = lds + (t & 1) * 2 * L::SIDE, *vt = kt + L::SIDE;
            const int first = wk * 32 * KS;                       // this wave's keys of the tile
            const int j0 = k0 + t * L::KEYS + first, j1 = j0 + 32 * KS - 1;
            if (idle || j0 > jhi_max || j1 < jlo_min) continue;   // none of them seen
            // scores
            f32x16 s[KS];
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
                for (int e = 0; e < 16; ++e) s[ks][e] = 0.0f;
                const int row = first + ks * 32 + l32, f = L::key_unit(row);
#pragma unroll
                for (int x = 0; x < NQ; ++x) {
                    const uint4 kf = *reinterpret_cast<const uint4 *>(kt + row * RB + (((2 * x + half) ^ f) << 4));
                    if constexpr (BF) {
                        s[ks] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                            __builtin_bit_cast(bf16x8_t, kf), __builtin_bit_cast(bf16x8_t, qf[x]), s[ks], 0, 0, 0);
                    } else {
                        const float4 ka = __builtin_bit_cast(float4, kf), qb = __builtin_bit_cast(float4, qf[x]);
                        s[ks] = __builtin_amdgcn_mfma_f32_32x32x2f32(ka.x, qb.x, s[ks], 0, 0, 0);
                        s[ks] = __builtin_amdgcn_mfma_f32_32x32x2f32(ka.y, qb.y, s[ks], 0, 0, 0);
                        s[ks] = __builtin_amdgcn_mfma_f32_32x32x2f32(ka.z, qb.z, s[ks], 0, 0, 0);
                        s[ks] = __builtin_amdgcn_mfma_f32_32x32x2f32(ka.w, qb.w, s[ks], 0, 0, 0);
                    }
                }
            }
            const bool masked = j1 > jhi_min || j0 < jlo_max;
            if (masked) {
#pragma unroll
                for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int j = j0 + ks * 32 + 8 * (e / 4) + 4 * half + e % 4;
                        s[ks][e] = j >= jlo && j <= jhi ? s[ks][e] : -INFINITY;
                    }
            }
            // the running maximum, moved only when a row's scores pass it by more than 2^8 (in the
            // weights p, which fp32 sums hold as well): what was summed is then scaled
            float top = s[0][0];
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int e = 0; e < 16; ++e) top = fmaxf(top, s[ks][e]);
            top = fmaxf(top, __shfl_xor(top, 32));
            if (__any(top * c > m * c + 8.0f)) {
                const float mn = fmaxf(m, top);
                const float alpha = mn == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m - mn) * c);
                l *= alpha;
#pragma unroll
                for (int d = 0; d < ND; ++d)
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[d][e] *= alpha;
                m = mn;
            }
            const float mc = m == -INFINITY ? 0.0f : m * c;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    s[ks][e] = __builtin_amdgcn_exp2f(fmaf(s[ks][e], c, -mc));
                    l += s[ks][e];
                }
            // O^T += V^T P^T
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const int row = first + ks * 32;
                if constexpr (BF) {
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        bf16x8_t p;
#pragma unroll
                        for (int e = 0; e < 8; ++e) p[e] = (__bf16)s[ks][8 * j + e];
                        // lane i of 16 reads four columns of key i / 4 and gets column i of four keys
                        const int i = lane & 15, key = row + 16 * j + 4 * half + i / 4;
                        const int f = L::value_unit(4 * half + i / 4);   // row and 16 j are multiples of 8
#pragma unroll
                        for (int d = 0; d < ND; ++d) {
                            const int u = d * 4 + ((lane >> 4) & 1) * 2 + ((i & 3) >> 1);
                            const unsigned char *at = vt + key * RB + ((u ^ f) << 4) + (i & 1) * 8;
                            typedef __attribute__((address_space(3))) s16x4 lds4;
                            const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(at));
                            const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(at + 8 * RB));
                            const s16x8 v = {v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
                            o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, v), p, o[d],
                                                                           0, 0, 0);
                        }
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int key = row + 8 * (e / 4) + 4 * half + e % 4, f = half << 3;
#pragma unroll
                        for (int d = 0; d < ND; ++d) {
                            const float v = *reinterpret_cast<const float *>(
                                vt + key * RB + (((d * 8 + l32 / 4) ^ f) << 4) + (l32 & 3) * 4);
                            o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, s[ks][e], o[d], 0, 0, 0);
                        }
                    }
                }
            }
        }
        l += __shfl_xor(l, 32);

        if constexpr (WK > 1) {   // the waves of the same rows join their sums
            __syncthreads();
            float *oj = reinterpret_cast<float *>(lds), *ml = oj + L::NW * 32 * DP;
            if (half == 0) {
                ml[w * 64 + l32] = m;
                ml[w * 64 + 32 + l32] = l;
            }
            __syncthreads();
            float mt = -INFINITY;
#pragma unroll
            for (int k = 0; k < WK; ++k) mt = fmaxf(mt, ml[(wr * WK + k) * 64 + l32]);
            const float m0 = mt == -INFINITY ? 0.0f : mt;
            float lt = 0.0f;
#pragma unroll
            for (int k = 0; k < WK; ++k)
                lt += ml[(wr * WK + k) * 64 + 32 + l32] *
                      __builtin_amdgcn_exp2f((ml[(wr * WK + k) * 64 + l32] - m0) * c);
            const float alpha = __builtin_amdgcn_exp2f((m - m0) * c);
            m = mt;
            l = lt;
            // [value of the row][row], so that a store's lanes fall on consecutive words
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    oj[(w * DP + d * 32 + 8 * (e / 4) + 4 * half + e % 4) * 32 + l32] = o[d][e] * alpha;
            __syncthreads();
            // wave wk takes the blocks of 32 values wk, wk + WK, ...
#pragma unroll
            for (int d = 0; d < ND; ++d)
                if (d % WK == wk) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int at = (d * 32 + 8 * (e / 4) + 4 * half + e % 4) * 32 + l32;
                        float sum = 0.0f;
#pragma unroll
                        for (int k = 0; k < WK; ++k) sum += oj[(wr * WK + k) * DP * 32 + at];
                        o[d][e] = sum;
                    }
                }
        }

        const long long orow = (long long)(q0 + qi) * a.kv_heads * a.group + head;
        if (stored && used > 1) {
            const long long at = orow * a.splits + split;
            float *po = a.part_o + at * a.dim;
#pragma unroll
            for (int d = 0; d < ND; ++d)
                if (WK == 1 || d % WK == wk)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int at0 = d * 32 + 8 * e + 4 * half;
                        if (at0 < a.dim)
                            *reinterpret_cast<float4 *>(po + at0) =
                                make_float4(o[d][4 * e], o[d][4 * e + 1], o[d][4 * e + 2], o[d][4 * e + 3]);
                    }
            if (wk == 0 && half == 0) {
                a.part_ml[at * 2] = m * c;
                a.part_ml[at * 2 + 1] = l;
            }
        } else if (stored) {
            const float inv = l == 0.0f ? 0.0f : 1.0f / l;   // a row that sees nothing is zero
            T *out = static_cast<T *>(a.o) + (long long)(q0 + qi) * a.os[0] + (long long)head * a.os[1];
#pragma unroll
            for (int d = 0; d < ND; ++d)
                if (WK == 1 || d % WK == wk)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int at0 = d * 32 + 8 * e + 4 * half;
                        if (at0 >= a.dim) continue;
                        if constexpr (BF) {
                            union { uint2 q; uint16_t e[4]; } v;
#pragma unroll
                            for (int x = 0; x < 4; ++x) v.e[x] = f32_to_bf16_rne(o[d][4 * e + x] * inv);
                            *reinterpret_cast<uint2 *>(out + at0) = v.q;
                        } else {
                            *reinterpret_cast<float4 *>(out + at0) =
                                make_float4(o[d][4 * e] * inv, o[d][4 * e + 1] * inv, o[d][4 * e + 2] * inv,
                                            o[d][4 * e + 3] * inv);
                        }
                    }
            if (a.lse && wk == 0 && half == 0)
                a.lse[orow] = l == 0.0f ? -INFINITY : (m * c + __log2f(l)) * 0.693147180559945309f;
        }
    }
}

template <typename T, int DP, int WR, int WK, int KS>
hipError_t attn_go(const AttnArgs &a, hipStream_t st) {
    using L = AttnTile<T, DP, WR, WK, KS>;
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void *>(attn_kernel<T, DP, WR, WK, KS>),
                                                       hipFuncAttributeMaxDynamicSharedMemorySize, L::LDS);
    if (attr != hipSuccess) return attr;
    const long long blocks = (long long)a.tiles * a.splits * a.kv_heads * a.batch;
    attn_kernel<T, DP, WR, WK, KS><<<(unsigned)blocks, L::THREADS, L::LDS, st>>>(a);
    return hipGetLastError();
}

}  // namespace ftcnn
