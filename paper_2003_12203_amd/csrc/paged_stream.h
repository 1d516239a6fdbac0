// Attention of a few rows over many cached keys (single new tokens, short chunks): the kernel.
//
// The mathematics, the units and the schedules are those of paged_attn.h.  What bounds it is the reading
// of keys and values, once each, so a wave works alone and keeps as much of it in flight as it can: a
// tile of 16 S2 keys goes from memory straight into registers, the next tile's keys as soon as this
// one's are multiplied, its values as soon as this one's are, and no wave waits for another.  Tiles of
// 16 x 16 leave registers for three or more waves on each SIMD.
//
// Loads are in the order of the matrix instructions' operands.  Keys: lane (n, h) = (lane % 16, lane / 16)
// takes unit 4 x + h (16 bytes) of key n: 64 bytes of a row at a time.  S^T = K Q^T leaves scores of row n
// and keys 4 h + i in that lane, which are also where O^T = V^T P^T wants its weights if the product
// takes one key a lane: that is the fp32 instruction (four keys), so that values are widened to fp32 in
// registers, weights are not rounded, and nothing is transposed: lane (m, h) takes the VE values from
// VE m on of key 4 h + i, a whole row in 16 lanes, one value of each for VE instructions.  At a quarter of the
// bf16 rate or less it still takes half the time of the loads.
//
// Measured with the join, bf16, 32 heads of 128 over eight key heads: one token over 131072, 537 MB, 116 us
// (105 without, 5.1 TB/s of the 5.2 that a large copy reaches); 64 single tokens over 204 MB of ragged caches 57 us (50
// without); through LDS in workgroups that share the loads the latter took 81.  fp32, the same: 228 us (1.07 GB) and 86
// (408 MB).  Over few keys the start is all: 76 keys
// 10.5 us, in which loads wait for each other: lengths, page list, keys, and the next tile's after this one's.
#pragma once

#include "paged_attn.h"

namespace ftcnn {

typedef float f32x4_t __attribute__((ext_vector_type(4)));

template <typename T, int DP> struct StreamTile {
    // keys of a tile: what 32 to 64 registers hold of keys, and of values
    static constexpr int S2 = DP * (int)sizeof(T) <= 256 ? 2 : 1, KEYS = 16 * S2;
    static constexpr int EU = 16 / sizeof(T), NQ = DP * (int)sizeof(T) / 64, VE = DP / 16;
    static constexpr int VB = VE * (int)sizeof(T) < 16 ? 8 : 16;            // bytes of a load of values
    static constexpr int VU = VE * (int)sizeof(T) / VB, VL = VB / sizeof(T);   // loads of a key, values of a load
};

template <typename T, int DP, bool EVEN>
__global__ __launch_bounds__(64, DP * sizeof(T) <= 128 ? 3 : DP * sizeof(T) <= 512 ? 2 : 1) void stream_kernel(AttnArgs a) {
    using L = StreamTile<T, DP>;
    constexpr bool BF = sizeof(T) == 2;
    constexpr int S2 = L::S2, KEYS = L::KEYS, EU = L::EU, NQ = L::NQ, VE = L::VE, VU = L::VU, VL = L::VL;
    constexpr int ROWS = 16;
    const int lane = threadIdx.x, n16 = lane & 15, h = lane >> 4;
    const float c = a.scale_log2;

    // As attn_schedule has it.
    auto unit = [&](const AttnSeq &sq, int b, int hk, int rt, int from, int to, long long part) __attribute__((always_inline)) {
        const int nrows = sq.nq * a.group, r0 = rt * ROWS;
        const int i0 = (int)div_by(r0, a.div_group), i1 = (int)div_by(min(r0 + ROWS, nrows) - 1, a.div_group);
        int lo, hi;
        sq.range(a, i0, i1, lo, hi);
        const int k0 = uniform(min(hi, lo + from)), k1 = uniform(to < hi - lo ? lo + to : hi);
        const int ntiles = k1 > k0 ? (k1 - k0 + KEYS - 1) / KEYS : 0;

        const char *kbase = static_cast<const char *>(a.k) + (long long)hk * a.kb[2];
        const char *vbase = static_cast<const char *>(a.v) + (long long)hk * a.vb[2];
        const int32_t *list = a.page_list + (long long)b * a.list_stride;
        // the page of key lane % KEYS of a tile
        auto key_of = [&](int t) { return min(k0 + t * KEYS + lane % KEYS, k1 - 1); };
        auto lookup = [&](int t) { return list[div_by(key_of(t), a.div_page)]; };
        uint4 kf[S2][NQ];
        auto load_k = [&](int t, int found) {
            const int pid = min(max(found, 0), a.pages - 1);
            const int key = key_of(t), in_page = key - (int)div_by(key, a.div_page) * a.page;
#pragma unroll
            for (int s = 0; s < S2; ++s) {
                const int p = __shfl(pid, 16 * s + n16), x = __shfl(in_page, 16 * s + n16);
                const T *row = reinterpret_cast<const T *>(kbase + page_row(p, a.kb[0], x, a.kb[1]));
#pragma unroll
                for (int q = 0; q < NQ; ++q) {
                    const int col = (4 * q + h) * EU;
                    kf[s][q] = *reinterpret_cast<const uint4 *>(row + (col < a.dim ? col : 0));
                }
            }
        };
        typedef typename std::conditional<L::VB == 8, uint2, uint4>::type VT;
        VT vf[S2][4][VU];
        auto load_v = [&](int t, int found) {
            const int pid = min(max(found, 0), a.pages - 1);
            const int key = key_of(t), in_page = key - (int)div_by(key, a.div_page) * a.page;
#pragma unroll
            for (int s = 0; s < S2; ++s)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int at = 16 * s + 4 * h + i, p = __shfl(pid, at), x = __shfl(in_page, at);
                    const T *row = reinterpret_cast<const T *>(vbase + page_row(p, a.vb[0], x, a.vb[1]));
#pragma unroll
                    for (int u = 0; u < VU; ++u) {
                        const int col = n16 * VE + u * VL;   // past the head: any values, of columns not stored
                        vf[s][i][u] = *reinterpret_cast<const VT *>(row + (col < a.dim ? col : 0));
                    }
                }
        };
        auto value = [&](int s, int i, int e) -> float {
            const VT &q = vf[s][i][e / VL];
            const uint32_t *w = reinterpret_cast<const uint32_t *>(&q);
            if constexpr (BF) {
                const uint32_t x = w[e % VL / 2];
                return __builtin_bit_cast(float, e % 2 ? x & 0xffff0000u : x << 16);
            } else {
                return __builtin_bit_cast(float, w[e % VL]);
            }
        };
        int pid = 0, pid1 = 0;
        if (ntiles > 0) {
            pid = lookup(0);
            if (ntiles > 1) pid1 = lookup(1);
            load_k(0, pid);
            load_v(0, pid);
        }
        // this lane's row; past the last one, the last again (not stored)
        const int mine = r0 + n16, r = min(mine, nrows - 1);
        const int qi = (int)div_by(r, a.div_group), head = hk * a.group + r - qi * a.group;
        const int pos = sq.kv - sq.nq + qi;
        const int jhi = min(a.causal ? pos : sq.kv - 1, k1 - 1);   // the keys it sees: jlo..jhi
        const int jlo = a.window > 0 ? pos - a.window + 1 : 0;
        const int jhi_min = __builtin_amdgcn_readlane(jhi, 0), jlo_max = __builtin_amdgcn_readlane(jlo, 15);
        uint4 qf[NQ];
        {
            const T *row = static_cast<const T *>(a.q) + (long long)(sq.q0 + qi) * a.qs[0] + (long long)head * a.qs[1];
#pragma unroll
            for (int q = 0; q < NQ; ++q) {
                const int col = (4 * q + h) * EU;
                qf[q] = col < a.dim ? *reinterpret_cast<const uint4 *>(row + col) : make_uint4(0, 0, 0, 0);
            }
        }
        f32x4_t o[VE];
#pragma unroll
        for (int e = 0; e < VE; ++e) o[e] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
        float m = -INFINITY, l = 0.0f;

        int dirt0 = INT_MAX, dirt1 = -1;   // the first and last tile with values not finite
        for (int t = 0; t < ntiles; ++t) {
            if (DP != a.dim) {   // keys' columns past the head: zero, as the queries' are
#pragma unroll
                for (int s = 0; s < S2; ++s)
#pragma unroll
                    for (int q = 0; q < NQ; ++q)
                        if ((4 * q + h) * EU >= a.dim) kf[s][q] = make_uint4(0, 0, 0, 0);
            }
            f32x4_t s[S2];
#pragma unroll
            for (int k = 0; k < S2; ++k) {
                s[k] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int q = 0; q < NQ; ++q) {
                    if constexpr (BF) {
                        s[k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                            __builtin_bit_cast(bf16x8_t, kf[k][q]), __builtin_bit_cast(bf16x8_t, qf[q]), s[k], 0, 0, 0);
                    } else {
                        const float4 ka = __builtin_bit_cast(float4, kf[k][q]);
                        const float4 qb = __builtin_bit_cast(float4, qf[q]);
                        s[k] = __builtin_amdgcn_mfma_f32_16x16x4f32(ka.x, qb.x, s[k], 0, 0, 0);
                        s[k] = __builtin_amdgcn_mfma_f32_16x16x4f32(ka.y, qb.y, s[k], 0, 0, 0);
                        s[k] = __builtin_amdgcn_mfma_f32_16x16x4f32(ka.z, qb.z, s[k], 0, 0, 0);
                        s[k] = __builtin_amdgcn_mfma_f32_16x16x4f32(ka.w, qb.w, s[k], 0, 0, 0);
                    }
                }
            }
            const int pid_next = pid1;
            if (t + 1 < ntiles) load_k(t + 1, pid_next);
            if (t + 2 < ntiles) pid1 = lookup(t + 2);
            const int j0 = k0 + t * KEYS;
            const bool masked = j0 + KEYS - 1 > jhi_min || j0 < jlo_max;
            if (masked) {
#pragma unroll
                for (int k = 0; k < S2; ++k)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int j = j0 + 16 * k + 4 * h + i;
                        s[k][i] = j >= jlo && j <= jhi ? s[k][i] : -INFINITY;
                    }
            }
            float top = s[0][0];
#pragma unroll
            for (int k = 0; k < S2; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i) top = fmaxf(top, s[k][i]);
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            // the running maximum, moved only when scores pass it by more than 2^8 (in the weights)
            if (__any(top * c > m * c + 8.0f)) {
                const float mn = fmaxf(m, top);
                const float alpha = mn == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m - mn) * c);
                l *= alpha;
#pragma unroll
                for (int e = 0; e < VE; ++e)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[e][i] *= alpha;
                m = mn;
            }
            const float mc = m == -INFINITY ? 0.0f : m * c;
#pragma unroll
            for (int k = 0; k < S2; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[k][i] = __builtin_amdgcn_exp2f(fmaf(s[k][i], c, -mc));
                    l += s[k][i];
                }
            if (masked) {   // see NonFinite
                bool any = false;
#pragma unroll
                for (int k = 0; k < S2; ++k)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int u = 0; u < VU; ++u)
#pragma unroll
                            for (int x = 0; x < L::VB / 4; ++x)
                                any |= wash<T>(reinterpret_cast<uint32_t *>(&vf[k][i][u])[x]);
                if (__any(any)) {
                    dirt0 = min(dirt0, t);
                    dirt1 = t;
                }
            }
#pragma unroll
            for (int k = 0; k < S2; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int e = 0; e < VE; ++e) {
                        const float v = value(k, i, e);
                        o[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, s[k][i], o[e], 0, 0, 0);
                    }
            if (t + 1 < ntiles) load_v(t + 1, pid_next);
        }

        for (int j = dirt0; j <= dirt1; ++j)
            for (int key = k0 + j * KEYS; key < min(k1, k0 + (j + 1) * KEYS); ++key) {
                const int in = (int)div_by(key, a.div_page), pg = min(max(list[in], 0), a.pages - 1);
                const T *row = reinterpret_cast<const T *>(vbase + page_row(pg, a.vb[0], key - in * a.page, a.vb[1]));
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int e = 0; e < VE; e += 4) {
                        const int d = VE * (4 * h + i) + e;   // past the head: any values, of columns not stored
                        const T *at = row + (d < a.dim ? d : 0);
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            const float v = value_of(at[x]);
                            o[e + x][i] += key >= jlo && key <= jhi && !(fabsf(v) < INFINITY) ? v : 0.0f;
                        }
                    }
            }
        float sum = l + __shfl_xor(l, 16);
        sum += __shfl_xor(sum, 32);
        if (mine >= nrows) return;
        // o[e][i] is value VE (4 h + i) + e of the row
        if (part >= 0) {
            const long long at = part * a.part_rows + (mine - r0);
            float *po = a.part_o + at * a.dim;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < VE; e += 4) {
                    const int d = VE * (4 * h + i) + e;
                    if (d < a.dim) store4(po + d, make_float4(o[e][i], o[e + 1][i], o[e + 2][i], o[e + 3][i]));
                }
            if (h == 0) {
                a.part_ml[at * 2] = m * c;
                a.part_ml[at * 2 + 1] = sum;
            }
            return;
        }
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;   // a row that sees nothing is zero
        T *out = static_cast<T *>(a.o) + (long long)(sq.q0 + qi) * a.os[0] + (long long)head * a.os[1];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < VE; e += 4) {
                const int d = VE * (4 * h + i) + e;
                if (d < a.dim)
                    store4(out + d, make_float4(o[e][i] * inv, o[e + 1][i] * inv, o[e + 2][i] * inv, o[e + 3][i] * inv));
            }
        if (a.lse && h == 0)
            a.lse[(long long)(sq.q0 + qi) * a.kv_heads * a.group + head] =
                sum == 0.0f ? -INFINITY : (m * c + __log2f(sum)) * 0.693147180559945309f;
    };
    attn_schedule<EVEN>(a, ROWS, KEYS, unit);
    attn_clear_unowned<T, 64>(a);
}

template <typename T, int DP> hipError_t stream_go(const AttnArgs &a, hipStream_t st) {
    if (a.groups) stream_kernel<T, DP, true><<<a.groups, 64, 0, st>>>(a);
    else stream_kernel<T, DP, false><<<(unsigned)a.tiles * a.kv_heads * a.batch, 64, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace ftcnn
