// The attention weight that every cached key gets from the new tokens:
//
//   mass_j += sum over rows i that see j of exp(scale q_i . k_j - L_i),
//
// with the rows' log-sums L given, so that the weights need no second pass over the keys.  Rows, sequences and masks
// are those of paged_attn.h.  The product is S^T = K Q^T: a lane has one row and several keys, whose weights it adds up
// over all rows and heads in registers; lanes are added at the end.  No order hangs on timing.
//
// mass_wide_kernel, more than 16 rows of a key head: a wave holds 32 KS keys of a head in registers, tiles of 64 rows
// (fewer where heads are large) go through LDS, which the workgroup's waves share.
// mass_few_kernel: the reading of the keys is all, straight into registers in the order of the matrix instructions; a
// wave takes every fourth head of a block of keys.
#pragma once

#include "mass.h"
#include "paged_stream.h"

namespace ftcnn {

// The first row tile that may see a key of [k0, k1), and the one behind the last, of tiles of `rows` rows.
__device__ __forceinline__ void rows_that_see(const AttnArgs &a, const AttnSeq &sq, int k0, int k1, int rows, int &t0, int &t1) {
    const int past = sq.kv - sq.nq;
    const int i0 = a.causal ? min(max(k0 - past, 0), sq.nq) : 0;                          // the first token
    const int i1 = a.window > 0 ? min(max(k1 - 1 - past + a.window, 0), sq.nq) : sq.nq;   // behind the last
    t0 = (int)((long long)i0 * a.group / rows);
    t1 = i1 > i0 ? (i1 * a.group + rows - 1) / rows : t0;
}

// This lane's row r (past the last one: sees nothing), what it sees, and where it is.
struct MassRow {
    int jlo, jhi, qi, head;
    __device__ __forceinline__ MassRow(const AttnArgs &a, const AttnSeq &sq, int hk, int r) {
        const int nrows = sq.nq * a.group, at = min(r, nrows - 1);
        qi = (int)div_by(at, a.div_group);
        head = hk * a.group + at - qi * a.group;
        const int pos = sq.kv - sq.nq + qi;
        jhi = r < nrows ? (a.causal ? pos : sq.kv - 1) : -1;
        jlo = a.window > 0 ? pos - a.window + 1 : 0;
    }
};

template <typename T, int DP, int KS>
__global__ __launch_bounds__(256, DP * sizeof(T) * KS <= 512 ? 2 : 1) void mass_wide_kernel(MassArgs p) {
    constexpr int QS = DP * (int)sizeof(T) <= 512 ? 2 : 1;   // row tiles of 32 in LDS at a time
    using L = AttnTile<T, DP, 4, QS>;
    constexpr bool BF = sizeof(T) == 2;
    constexpr int UPR = L::UPR, EU = L::EU, RB = L::RB, NQ = UPR / 2, ROWS = L::KEYS, KEYS = 128 * KS;
    constexpr int OWN = ROWS / 4, STEP = 64 / UPR;
    extern __shared__ __align__(1024) unsigned char lds[];
    const AttnArgs &a = p.t;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, half = lane >> 5;
    typedef __attribute__((address_space(3))) unsigned char lds_byte;
    const unsigned lds_at = (unsigned)(uintptr_t)(lds_byte *)lds;
    const float c = a.scale_log2;
    if (DP != a.dim)   // the columns past the head, which no load writes
        for (int i = tid; i < 2 * L::SIDE / 16; i += 256) reinterpret_cast<uint4 *>(lds)[i] = make_uint4(0, 0, 0, 0);
    unsigned x = blockIdx.x;
    const int hp = (int)(x % (unsigned)p.head_parts);
    x /= (unsigned)p.head_parts;
    const int b = (int)(x % (unsigned)a.batch);
    x /= (unsigned)a.batch;
    const int rp = (int)(x % (unsigned)p.row_parts);
    const int h0 = a.kv_heads * hp / p.head_parts, h1 = a.kv_heads * (hp + 1) / p.head_parts;
    AttnSeq sq(a, b, ROWS);
    sq.settle();
    const int32_t *list = a.page_list + (long long)b * a.list_stride;
    const int nrows = sq.nq * a.group;
    const int own = lane / UPR, slot = lane % UPR;

    for (int kb = (int)(x / (unsigned)p.row_parts); (long long)kb * KEYS < sq.kv; kb += p.blocks) {
        const int k0 = kb * KEYS + w * 32 * KS;   // this wave's keys
        int t0, t1;
        rows_that_see(a, sq, kb * KEYS, min(kb * KEYS + KEYS, sq.kv), ROWS, t0, t1);
        const int some = (t1 - t0 + p.row_parts - 1) / p.row_parts;
        t0 = uniform(min(t0 + rp * some, t1));
        t1 = uniform(min(t0 + some, t1));
        float acc[KS][16];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[ks][e] = 0.0f;
        const char *krow[KS];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {   // past the last key that one again, which counts nowhere
            const int key = min(k0 + 32 * ks + l32, sq.kv - 1), in = (int)div_by(key, a.div_page);
            krow[ks] = static_cast<const char *>(a.k) +
                       page_row(min(max(list[in], 0), a.pages - 1), a.kb[0], key - in * a.page, a.kb[1]);
        }
        for (int hk = h0; hk < h1 && t1 > t0; ++hk) {
            uint4 kf[KS][NQ];
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int q = 0; q < NQ; ++q) {
                    const int u = 2 * q + half;
                    kf[ks][q] = u * EU < a.dim ? *reinterpret_cast<const uint4 *>(krow[ks] + (long long)hk * a.kb[2] + u * 16)
                                               : make_uint4(0, 0, 0, 0);
                }
            auto issue = [&](int t) __attribute__((always_inline)) {   // rows of tile t into half t % 2 of LDS
#pragma unroll
                for (int i = 0; i < L::LOADS; ++i) {
                    const int row = w * OWN + own + i * STEP, u = slot ^ L::key_unit(row);
                    if (DP != a.dim && u * EU >= a.dim) continue;
                    const int at = min(t * ROWS + row, nrows - 1), qi = (int)div_by(at, a.div_group);
                    const T *from = static_cast<const T *>(a.q) + (long long)(sq.q0 + qi) * a.qs[0] +
                                    (long long)(hk * a.group + at - qi * a.group) * a.qs[1];
                    load_to_lds(reinterpret_cast<const char *>(from) + u * 16,
                                lds_at + (t & 1) * L::SIDE + w * OWN * RB + i * 1024);
                }
            };
            float next[QS];
            auto logs = [&](int t) __attribute__((always_inline)) {
#pragma unroll
                for (int s = 0; s < QS; ++s) {
                    const MassRow row(a, sq, hk, t * ROWS + 32 * s + l32);
                    next[s] = p.lse[(long long)(sq.q0 + row.qi) * a.kv_heads * a.group + row.head];
                }
            };
            __syncthreads();   // the head before this one has been read
            issue(t0);
            logs(t0);
            for (int t = t0; t < t1; ++t) {
                wait_loads();
                tile_barrier();   // tile t has landed, and nobody reads tile t - 1 any more
                float log2e[QS];
#pragma unroll
                for (int s = 0; s < QS; ++s) log2e[s] = next[s] * 1.44269504088896340736f;
                if (t + 1 < t1) {
                    issue(t + 1);
                    logs(t + 1);
                }
                // do all rows of the tile see all of this wave's keys?
                const int i0 = (int)div_by(t * ROWS, a.div_group);
                const int i1 = (int)div_by(min((t + 1) * ROWS, nrows) - 1, a.div_group);
                const bool whole = (t + 1) * ROWS <= nrows && k0 + 32 * KS <= sq.kv &&
                                   (!a.causal || sq.kv - sq.nq + i0 >= k0 + 32 * KS - 1) &&
                                   (a.window == 0 || sq.kv - sq.nq + i1 - a.window + 1 <= k0);
#pragma unroll
                for (int s = 0; s < QS; ++s) {
                    f32x16 sc[KS];
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                        for (int e = 0; e < 16; ++e) sc[ks][e] = 0.0f;
                    const int row = 32 * s + l32, f = L::key_unit(row);
                    const unsigned char *at = lds + (t & 1) * L::SIDE + row * RB;
#pragma unroll
                    for (int q = 0; q < NQ; ++q) {
                        const uint4 qf = *reinterpret_cast<const uint4 *>(at + (((2 * q + half) ^ f) << 4));
#pragma unroll
                        for (int ks = 0; ks < KS; ++ks) {
                            if constexpr (BF) {
                                sc[ks] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                                    __builtin_bit_cast(bf16x8_t, kf[ks][q]), __builtin_bit_cast(bf16x8_t, qf), sc[ks], 0, 0, 0);
                            } else {
                                const float4 ka = __builtin_bit_cast(float4, kf[ks][q]), qb = __builtin_bit_cast(float4, qf);
                                sc[ks] = __builtin_amdgcn_mfma_f32_32x32x2f32(ka.x, qb.x, sc[ks], 0, 0, 0);
                                sc[ks] = __builtin_amdgcn_mfma_f32_32x32x2f32(ka.y, qb.y, sc[ks], 0, 0, 0);
                                sc[ks] = __builtin_amdgcn_mfma_f32_32x32x2f32(ka.z, qb.z, sc[ks], 0, 0, 0);
                                sc[ks] = __builtin_amdgcn_mfma_f32_32x32x2f32(ka.w, qb.w, sc[ks], 0, 0, 0);
                            }
                        }
                    }
                    if (whole) {
#pragma unroll
                        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                            for (int e = 0; e < 16; ++e)
                                acc[ks][e] += __builtin_amdgcn_exp2f(fmaf(sc[ks][e], c, -log2e[s]));
                    } else {
                        const MassRow mine(a, sq, hk, t * ROWS + row);
                        const int jhi = min(mine.jhi, sq.kv - 1);
#pragma unroll
                        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                            for (int e = 0; e < 16; ++e) {
                                const int j = k0 + 32 * ks + 8 * (e / 4) + 4 * half + e % 4;
                                const float v = __builtin_amdgcn_exp2f(fmaf(sc[ks][e], c, -log2e[s]));
                                acc[ks][e] += j >= mine.jlo && j <= jhi ? v : 0.0f;
                            }
                    }
                }
            }
        }
        const int part = hp * p.row_parts + rp;
        const bool alone = p.head_parts * p.row_parts == 1;
        float *to = alone ? p.mass + b * p.mass_stride : p.part + ((long long)part * a.batch + b) * a.capacity;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                float v = acc[ks][e];
#pragma unroll
                for (int x = 1; x < 32; x *= 2) v += __shfl_xor(v, x);
                const int j = k0 + 32 * ks + 8 * (e / 4) + 4 * half + e % 4;
                if (l32 == 0 && j < sq.kv) to[j] = alone ? to[j] + v : v;
            }
    }
}

template <typename T, int DP>
__global__ __launch_bounds__(256) void mass_few_kernel(MassArgs p) {
    using L = StreamTile<T, DP>;
    constexpr bool BF = sizeof(T) == 2;
    constexpr int S2 = L::S2, KEYS = L::KEYS, EU = L::EU, NQ = L::NQ, TILES = 4, BLOCK = KEYS * TILES;
    __shared__ float sums[4][BLOCK];
    const AttnArgs &a = p.t;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n16 = lane & 15, h = lane >> 4;
    const float c = a.scale_log2;
    const int b = (int)(blockIdx.x % (unsigned)a.batch);
    AttnSeq sq(a, b, 16);
    sq.settle();
    const int32_t *list = a.page_list + (long long)b * a.list_stride;
    for (int kb = (int)(blockIdx.x / (unsigned)a.batch); (long long)kb * BLOCK < sq.kv; kb += p.blocks) {
        const int k0 = kb * BLOCK, k1 = min(k0 + BLOCK, sq.kv);
        int r0, r1;
        rows_that_see(a, sq, k0, k1, 16, r0, r1);
        r0 = uniform(r0);
        r1 = uniform(r1);
        if (r1 <= r0) continue;   // (the same for all waves)
        const char *krow[TILES][S2];
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int s = 0; s < S2; ++s) {   // past the last key that one again, which counts nowhere
                const int key = min(k0 + t * KEYS + 16 * s + n16, sq.kv - 1), in = (int)div_by(key, a.div_page);
                krow[t][s] = static_cast<const char *>(a.k) +
                             page_row(min(max(list[in], 0), a.pages - 1), a.kb[0], key - in * a.page, a.kb[1]);
            }
        f32x4_t acc[TILES][S2];
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int s = 0; s < S2; ++s) acc[t][s] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
        for (int hk = w; hk < a.kv_heads; hk += 4)
            for (int rt = r0; rt < r1; ++rt) {
                const MassRow row(a, sq, hk, rt * 16 + n16);
                uint4 qf[NQ];
                const T *qrow = static_cast<const T *>(a.q) + (long long)(sq.q0 + row.qi) * a.qs[0] + (long long)row.head * a.qs[1];
#pragma unroll
                for (int q = 0; q < NQ; ++q) {
                    const int col = (4 * q + h) * EU;
                    qf[q] = col < a.dim ? *reinterpret_cast<const uint4 *>(qrow + col) : make_uint4(0, 0, 0, 0);
                }
                const float log2e = p.lse[(long long)(sq.q0 + row.qi) * a.kv_heads * a.group + row.head] * 1.44269504088896340736f;
                const int jhi = min(row.jhi, sq.kv - 1);
#pragma unroll
                for (int t = 0; t < TILES; ++t) {
                    if (k0 + t * KEYS >= k1) break;
                    uint4 kf[S2][NQ];
#pragma unroll
                    for (int s = 0; s < S2; ++s)
#pragma unroll
                        for (int q = 0; q < NQ; ++q) {
                            const int col = (4 * q + h) * EU;
                            kf[s][q] = col < a.dim ? *reinterpret_cast<const uint4 *>(krow[t][s] + (long long)hk * a.kb[2] + col * sizeof(T))
                                                   : make_uint4(0, 0, 0, 0);
                        }
#pragma unroll
                    for (int s = 0; s < S2; ++s) {
                        f32x4_t sc = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                        for (int q = 0; q < NQ; ++q) {
                            if constexpr (BF) {
                                sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                                    __builtin_bit_cast(bf16x8_t, kf[s][q]), __builtin_bit_cast(bf16x8_t, qf[q]), sc, 0, 0, 0);
                            } else {
                                const float4 ka = __builtin_bit_cast(float4, kf[s][q]), qb = __builtin_bit_cast(float4, qf[q]);
                                sc = __builtin_amdgcn_mfma_f32_16x16x4f32(ka.x, qb.x, sc, 0, 0, 0);
                                sc = __builtin_amdgcn_mfma_f32_16x16x4f32(ka.y, qb.y, sc, 0, 0, 0);
                                sc = __builtin_amdgcn_mfma_f32_16x16x4f32(ka.z, qb.z, sc, 0, 0, 0);
                                sc = __builtin_amdgcn_mfma_f32_16x16x4f32(ka.w, qb.w, sc, 0, 0, 0);
                            }
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int j = k0 + t * KEYS + 16 * s + 4 * h + i;
                            const float v = __builtin_amdgcn_exp2f(fmaf(sc[i], c, -log2e));
                            acc[t][s][i] += j >= row.jlo && j <= jhi ? v : 0.0f;
                        }
                    }
                }
            }
        __syncthreads();   // the block before this one has been read
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int s = 0; s < S2; ++s)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float v = acc[t][s][i];
#pragma unroll
                    for (int x = 1; x < 16; x *= 2) v += __shfl_xor(v, x);
                    if (n16 == 0) sums[w][t * KEYS + 16 * s + 4 * h + i] = v;
                }
        __syncthreads();
        float *to = p.mass + b * p.mass_stride;
        for (int j = threadIdx.x; j < k1 - k0; j += 256)
            to[k0 + j] += ((sums[0][j] + sums[1][j]) + sums[2][j]) + sums[3][j];
    }
}

template <typename T, int DP> hipError_t mass_go(const MassPlan &pl, const MassArgs &a, hipStream_t st) {
    const unsigned blocks = (unsigned)pl.blocks * a.t.batch * pl.head_parts * pl.row_parts;
    if (!pl.wide) {
        mass_few_kernel<T, DP><<<blocks, 256, 0, st>>>(a);
        return hipGetLastError();
    }
    constexpr int KS = DP * sizeof(T) <= 256 ? 2 : 1;
    constexpr int LDS = 2 * AttnTile<T, DP, 4, (DP * sizeof(T) <= 512 ? 2 : 1)>::SIDE;
    auto kernel = mass_wide_kernel<T, DP, KS>;
    if constexpr (LDS > 65536) {
        static std::atomic<uint64_t> raised{0};
        const hipError_t err = raise_lds_limit(reinterpret_cast<const void *>(kernel), LDS, raised);
        if (err != hipSuccess) return err;
    }
    kernel<<<blocks, 256, LDS, st>>>(a);
    return hipGetLastError();
}
template <typename T> hipError_t mass_pick(const MassPlan &pl, const MassArgs &a, hipStream_t st) {
    if (pl.dp == 64) return mass_go<T, 64>(pl, a, st);
    if (pl.dp == 128) return mass_go<T, 128>(pl, a, st);
    return mass_go<T, 256>(pl, a, st);
}

}  // namespace ftcnn
