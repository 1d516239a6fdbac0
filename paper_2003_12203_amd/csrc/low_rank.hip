// Low-rank adapters of many requests beside a shared projection:
//
//   out_t = y_t + s_a B_a (A_a x_t),  a = ids[t],  A_a [rank][ch], B_a [m][rank],
//
// in two launches, each a matrix product with tiles of tokens: h = A x with the channels split over waves
// and workgroups, whose sums are parts in the workspace, and out = y + B (s h), which adds the parts in
// their order.  A tile's tokens may have any adapters: its workgroups go over the different ones, each
// with the tokens that have it, the others' rows switched off.
#include <math.h>

#include <algorithm>

#include "low_rank.h"

namespace ftcnn {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Operands of 16 x 16 products come in units of 16 bytes: lane (n, h) = (lane % 16, lane / 16) holds unit
// h of row n, 64 bytes of a row in all (a chunk).  Both operands have the same order of values.
template <typename T> struct Chunk {
    static constexpr int EU = 16 / sizeof(T), VALUES = 4 * EU;
};
template <typename T> __device__ __forceinline__ f32x4 product(uint4 a, uint4 b, f32x4 c) {
    if constexpr (sizeof(T) == 2) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    } else {
        const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i], y[i], c, 0, 0, 0);
        return c;
    }
}

// Calls f(adapter, its tokens as bits) for the adapters of a tile of up to 64 tokens that fall to way `way` of
// `ways`; returns the bits of the tokens that have none.  By a whole wave.
template <typename F>
__device__ __forceinline__ unsigned long long each_adapter(const LowRankArgs &a, int t0, int tile, int way, int ways, F f) {
    const int lane = threadIdx.x & 63, count = min(tile, a.tokens - t0);
    int id = -1;
    if (lane < count) {
        id = a.ids[t0 + lane];
        if ((unsigned)id >= (unsigned)a.adapters) id = -1;
    }
    unsigned long long left = __ballot(id >= 0);
    const unsigned long long none = __ballot(lane < count && id < 0);
    for (int k = 0; left; k = k + 1 == ways ? 0 : k + 1) {
        const int adapter = __builtin_amdgcn_readlane(id, __builtin_ctzll(left));
        const unsigned long long mine = __ballot(id == adapter);
        left &= ~mine;
        if (k == way) f(adapter, mine);
    }
    return none;
}
__device__ __forceinline__ int used_rank(const LowRankArgs &a, int adapter) {
    return a.ranks ? min(max(a.ranks[adapter], 0), a.rank) : a.rank;
}

template <typename T, int MT, int NB>
__global__ __launch_bounds__(256) void shrink_kernel(LowRankArgs a) {
    using C = Chunk<T>;
    constexpr int TILE = 16 * MT, RANK = 16 * NB, AHEAD = MT + NB <= 3 ? 8 : (MT + NB <= 6 ? 4 : 2);
    __shared__ float sums[4][TILE][RANK];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n16 = lane & 15, h = lane >> 4;
    const unsigned split = blockIdx.x % (unsigned)a.splits, rest = blockIdx.x / (unsigned)a.splits;
    const int way = (int)(rest % (unsigned)a.ways), t0 = (int)(rest / (unsigned)a.ways) * TILE;
    const int chunks = (a.ch + C::VALUES - 1) / C::VALUES, runs = 4 * a.splits, run = (int)split * 4 + w;
    const int c0 = (int)((long long)chunks * run / runs), c1 = (int)((long long)chunks * (run + 1) / runs);
    each_adapter(a, t0, TILE, way, a.ways, [&](int adapter, unsigned long long mine) {
        const int rank = used_rank(a, adapter);
        const T *xr[MT], *ar[NB];
        bool xon[MT], aon[NB];
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            xon[i] = mine >> (16 * i + n16) & 1;
            xr[i] = static_cast<const T *>(a.x) + (long long)(t0 + 16 * i + n16) * a.xs + h * C::EU;
        }
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            aon[j] = 16 * j + n16 < rank;
            ar[j] = static_cast<const T *>(a.a) + adapter * a.as[0] + (16 * j + n16) * a.as[1] + h * C::EU;
        }
        f32x4 acc[MT][NB];
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        for (int c = c0; c < c1; c += AHEAD) {
            uint4 xf[AHEAD][MT], af[AHEAD][NB];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const int at = (c + k) * C::VALUES;
                const bool on = c + k < c1 && at + h * C::EU < a.ch;
#pragma unroll
                for (int i = 0; i < MT; ++i)
                    xf[k][i] = on && xon[i] ? *reinterpret_cast<const uint4 *>(xr[i] + at) : make_uint4(0, 0, 0, 0);
#pragma unroll
                for (int j = 0; j < NB; ++j)
                    af[k][j] = on && aon[j] ? *reinterpret_cast<const uint4 *>(ar[j] + at) : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int j = 0; j < NB; ++j) acc[i][j] = product<T>(xf[k][i], af[k][j], acc[i][j]);
        }
        // rows 4 h + e of tokens, column n16 of the rank
        __syncthreads();   // the adapter before this one
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) sums[w][16 * i + 4 * h + e][16 * j + n16] = acc[i][j][e];
        __syncthreads();
        const float s = a.scales ? a.scales[adapter] : 1.0f;
        for (int i = threadIdx.x; i < TILE * RANK; i += 256) {
            const int t = i / RANK, r = i % RANK;
            if (!(mine >> t & 1) || r >= a.rank) continue;
            a.part[((long long)split * a.tokens + t0 + t) * a.rank + r] =
                s * (((sums[0][t][r] + sums[1][t][r]) + sums[2][t][r]) + sums[3][t][r]);
        }
    });
}

// Unit k..k + EU of a row of B, without what lies past the rank that is used.
template <typename T> __device__ __forceinline__ uint4 within_rank(uint4 v, int k, int rank) {
    constexpr int EU = 16 / sizeof(T);
    union { uint4 q; T e[EU]; } u;
    u.q = v;
#pragma unroll
    for (int i = 0; i < EU; ++i)
        if (k + i >= rank) u.e[i] = 0;
    return u.q;
}

template <typename T> union Row16 {
    uint4 q[sizeof(T)];
    T e[16];
};
__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(uint16_t v) { return bf16_bits_to_f32(v); }
__device__ __forceinline__ void narrow(float &d, float v) { d = v; }
__device__ __forceinline__ void narrow(uint16_t &d, float v) { d = f32_to_bf16_rne(v); }

// The product is O^T = B H^T: a lane has a token, and of each of four blocks of 16 outputs the rows 4 h + e.
// Row 4 g + e of block q is output 16 g + 4 q + e, so that a lane's 16 values are neighbours and four lanes hold 64
// outputs of a token.
//
// bf16: h is taken as the sum of two bf16 values (an error of 2^-17 of it; rounded to one, its products would be off by as
// much as the outputs' own rounding).
template <typename T, int MT>
__global__ __launch_bounds__(256) void expand_kernel(LowRankArgs a) {
    using C = Chunk<T>;
    constexpr int EU = C::EU, TILE = 16 * MT, PLANES = sizeof(T) == 2 ? 2 : 1;
    constexpr int ROW = 128 + EU;   // values of a row: its units fall on different banks
    __shared__ __align__(16) T low[PLANES][TILE][ROW];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n16 = lane & 15, h = lane >> 4;
    const int groups = (a.m + a.columns - 1) / a.columns;
    const unsigned rest = blockIdx.x / (unsigned)groups;
    const int m0 = (int)(blockIdx.x % (unsigned)groups) * a.columns, m1 = min(m0 + a.columns, a.m);
    const int way = (int)(rest % (unsigned)a.expand_ways), t0 = (int)(rest / (unsigned)a.expand_ways) * TILE;
    const int chunks = (a.rank + C::VALUES - 1) / C::VALUES, full = chunks * C::VALUES;
    const unsigned long long none = each_adapter(a, t0, TILE, way, a.expand_ways, [&](int adapter, unsigned long long mine) {
        const int rank = used_rank(a, adapter);
        __syncthreads();   // the adapter before this one
        for (int i = threadIdx.x; i < TILE * full; i += 256) {
            const int t = i / full, r = i % full;
            float v = 0.0f;
            if (r < rank && mine >> t & 1)
                for (int s = 0; s < a.splits; ++s) v += a.part[((long long)s * a.tokens + t0 + t) * a.rank + r];
            if constexpr (PLANES == 2) {
                const uint16_t hi = f32_to_bf16_rne(v);
                low[0][t][r] = hi;
                // (of an infinity or NaN there is no rest)
                low[1][t][r] = fabsf(bf16_bits_to_f32(hi)) < INFINITY ? f32_to_bf16_rne(v - bf16_bits_to_f32(hi)) : 0;
            } else {
                low[0][t][r] = v;
            }
        }
        __syncthreads();
        for (int m = m0 + 64 * w; m < m1; m += 256) {
            f32x4 acc[4][MT];
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int i = 0; i < MT; ++i) acc[q][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            for (int c = 0; c < chunks; ++c) {
                const int k = c * C::VALUES + h * EU;
                uint4 bf[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int row = m + 16 * (n16 >> 2) + 4 * q + (n16 & 3);
                    bf[q] = make_uint4(0, 0, 0, 0);
                    if (row < a.m && k < rank) {
                        bf[q] = *reinterpret_cast<const uint4 *>(static_cast<const T *>(a.b) + adapter * a.bs[0] +
                                                                 row * a.bs[1] + k);
                        if (k + EU > rank) bf[q] = within_rank<T>(bf[q], k, rank);
                    }
                }
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int p = 0; p < PLANES; ++p) {
                        const uint4 hf = *reinterpret_cast<const uint4 *>(&low[p][16 * i + n16][k]);
#pragma unroll
                        for (int q = 0; q < 4; ++q) acc[q][i] = product<T>(bf[q], hf, acc[q][i]);
                    }
            }
            const int at = m + 16 * h;
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                if (!(mine >> (16 * i + n16) & 1)) continue;
                const long long t = t0 + 16 * i + n16;
                const T *y = static_cast<const T *>(a.y) + t * a.ys + at;
                T *out = static_cast<T *>(a.out) + t * a.os + at;
                Row16<T> v;
#pragma unroll
                for (int u = 0; u < (int)sizeof(T); ++u)
                    if (at + u * EU < a.m) v.q[u] = reinterpret_cast<const uint4 *>(y)[u];
#pragma unroll
                for (int e = 0; e < 16; ++e) narrow(v.e[e], widen(v.e[e]) + acc[e / 4][i][e % 4]);
#pragma unroll
                for (int u = 0; u < (int)sizeof(T); ++u)
                    if (at + u * EU < a.m) reinterpret_cast<uint4 *>(out)[u] = v.q[u];
            }
        }
    });
    if (way != 0 || a.out == a.y) return;
    for (unsigned long long left = none; left; left &= left - 1) {   // tokens without an adapter: as they are
        const long long t = t0 + __builtin_ctzll(left);
        const T *y = static_cast<const T *>(a.y) + t * a.ys;
        T *out = static_cast<T *>(a.out) + t * a.os;
        for (int c = m0 + EU * threadIdx.x; c < m1; c += EU * 256)
            *reinterpret_cast<uint4 *>(out + c) = *reinterpret_cast<const uint4 *>(y + c);
    }
}

template <typename T, int MT> hipError_t go(const LowRankArgs &a, hipStream_t st) {
    const unsigned blocks = (unsigned)a.tiles * a.ways * a.splits;
    if (a.rank <= 16) shrink_kernel<T, MT, 1><<<blocks, 256, 0, st>>>(a);
    else if (a.rank <= 32) shrink_kernel<T, MT, 2><<<blocks, 256, 0, st>>>(a);
    else if (a.rank <= 64) shrink_kernel<T, MT, 4><<<blocks, 256, 0, st>>>(a);
    else if constexpr (MT <= 2) shrink_kernel<T, MT, 8><<<blocks, 256, 0, st>>>(a);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    const unsigned groups = (unsigned)((a.m + a.columns - 1) / a.columns);
    expand_kernel<T, MT><<<(unsigned)a.tiles * a.expand_ways * groups, 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace

LowRankPlan low_rank_plan(const ftcnn_low_rank_desc &d) {
    LowRankPlan p{};
    if (d.tokens == 0) return p;
    p.tile = d.tokens <= 256 ? 16 : (d.rank <= 64 ? 64 : 32);
    p.tiles = (d.tokens + p.tile - 1) / p.tile;
    const int most = std::max(1, std::min(p.tile, d.adapters));
    const int chunks = (int)(((long long)d.ch * (d.dtype == FTCNN_F32 ? 4 : 2) + 63) / 64);
    const long long fill = 2 * kComputeUnits;
    auto share = [&](long long x) { return (int)std::max(1LL, std::min<long long>(most, fill / std::max(1LL, x))); };
    p.ways = share(p.tiles);
    // a wave has eight chunks at least
    p.splits = (int)std::max(1LL, std::min<long long>((chunks + 31) / 32, fill / ((long long)p.tiles * p.ways)));
    p.columns = 256;
    p.expand_ways = share((long long)p.tiles * ((d.m + 255) / 256) / 4);
    while ((long long)p.tiles * p.expand_ways * ((d.m + p.columns - 1) / p.columns) > 4 * fill && p.columns < 1024) p.columns *= 2;
    p.bytes = ((size_t)p.splits * d.tokens * d.rank * sizeof(float) + 255) & ~size_t(255);
    return p;
}

hipError_t launch_low_rank(int dtype, const LowRankPlan &pl, const LowRankArgs &a, hipStream_t st) {
    if (dtype == FTCNN_F32) {
        if (pl.tile == 16) return go<float, 1>(a, st);
        return pl.tile == 32 ? go<float, 2>(a, st) : go<float, 4>(a, st);
    }
    if (pl.tile == 16) return go<uint16_t, 1>(a, st);
    return pl.tile == 32 ? go<uint16_t, 2>(a, st) : go<uint16_t, 4>(a, st);
}

}  // namespace ftcnn
