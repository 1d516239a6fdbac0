// Norms of queries and keys for each head with the rotation by position, and keys and values
// written to a paged cache with the same on the way.
//
// A row is one head of one token: y = x * rsqrt(mean(x^2) + eps) * weight (with a weight), then
// every pair (a, b) of its first `rot` values becomes (a cos - b sin, b cos + a sin); the rest of
// the row is kept.  In fp32, rounded once.  Pairs are (i, i + rot/2) ("half") or (2i, 2i + 1)
// ("interleaved"); (cos, sin) of a pair at a position come from a table made once in float64.
//
// Memory-bound: a row is read and written once, and the table's row once for several heads.  A row is
// cut into units of two vectors of V values (16 bytes each, or fewer where alignment asks for it): a rotated
// unit holds V whole pairs, so a rotation needs no other lane.  A group of lanes holds a row, a unit or
// more a lane, and walks some heads of a token.
//
// Measured, 8192 tokens of 40 heads of 128 in bf16, normed and rotated, 172 MB: 37.7 us, 4.6 TB/s of the 5.2
// that a large copy reaches (vectors of four 44.5); 16384 tokens of eight such heads appended, 143 MB: 28.6 us.
// For few tokens the call's own time on the host, 7 to 10 us, is all.
#include <algorithm>

#include "paged.h"

namespace ftcnn {
namespace {

template <typename T, int V> struct Vec;
template <> struct Vec<float, 4> { typedef uint32_t type __attribute__((ext_vector_type(4))); };
template <> struct Vec<uint16_t, 8> { typedef uint32_t type __attribute__((ext_vector_type(4))); };
template <> struct Vec<uint16_t, 4> { typedef uint32_t type __attribute__((ext_vector_type(2))); };
template <> struct Vec<float, 1> { typedef float type; };
template <> struct Vec<uint16_t, 1> { typedef uint16_t type; };

template <typename T, int V> union Pack {
    typename Vec<T, V>::type q;
    T e[V];
};

__device__ inline float as_f32(float v) { return v; }
__device__ inline float as_f32(uint16_t v) { return bf16_bits_to_f32(v); }
__device__ inline void put(float &d, float v) { d = v; }
__device__ inline void put(uint16_t &d, float v) { d = f32_to_bf16_rne(v); }

// Rows in flight: bf16 two (16384 tokens appended 28.6 us, one 29.3), fp32 one (2049 tokens of 32 heads of 96,
// 10.6 us; two 11.4).
template <typename T> constexpr int kRowsInFlight = sizeof(T) == 2 ? 2 : 1;

// The sum over the LPR lanes of a group, in all of them: within rows of 16 lanes by the vector unit alone.
template <int CTRL> __device__ inline float with_lane(float x) {
    return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
template <int LPR> __device__ inline float group_sum(float x) {
    x = with_lane<0xB1>(x);                            // lane ^ 1
    x = with_lane<0x4E>(x);                            // lane ^ 2
    if constexpr (LPR >= 8) x = with_lane<0x141>(x);   // the other four of eight
    if constexpr (LPR >= 16) x = with_lane<0x140>(x);  // the other eight of sixteen
    if constexpr (LPR >= 32) x += __shfl_xor(x, 16, LPR);
    if constexpr (LPR >= 64) x += __shfl_xor(x, 32, LPR);
    return x;
}

// LPR lanes hold a row, UPL units a lane (unit lane + u * LPR).
template <typename T, int V, int LPR, int UPL, bool PAST_L2>
__global__ __launch_bounds__(kThreads, 4) void rope_kernel(RopeArgs a) {
    constexpr int B = UPL == 1 ? kRowsInFlight<T> : 1;
    const int lane = threadIdx.x % LPR;
    const unsigned id = blockIdx.x * (kThreads / LPR) + threadIdx.x / LPR;
    const unsigned token = div_by(id, a.div_chunks);
    int chunk = (int)(id - token * (unsigned)a.all_chunks);
    if (token >= (unsigned)a.tokens) return;
    int sec = 0;
    while (chunk >= a.chunks[sec]) chunk -= a.chunks[sec++];   // all_chunks is their sum
    const T *x = static_cast<const T *>(a.x[sec]) + (long long)token * a.xs[sec][0];
    T *y = static_cast<T *>(a.y[sec]);
    long long yh = a.ys[sec][1];
    if (a.slots) {
        const int64_t slot = a.slots[token];
        if (slot < 0 || slot >= (int64_t)a.pages * a.page) return;   // written nowhere
        const int64_t pg = slot / a.page;
        y += pg * a.ys[sec][0] + (slot - pg * a.page) * a.ys[sec][1];
        yh = a.ys[sec][2];
    } else {
        y += (long long)token * a.ys[sec][0];
    }
    const bool normed = sec < 2 && a.weight[sec];
    const bool rotated = sec < 2 && a.positions;
    const int units = a.dim / (2 * V), turned = rotated ? a.rot / (2 * V) : 0;
    int offa[UPL], offb[UPL];
    bool mine[UPL];
    float cs[UPL][2 * V], w[UPL][2 * V];
#pragma unroll
    for (int u = 0; u < UPL; ++u) {
        const int k = lane + u * LPR;
        mine[u] = k < units;
        const bool half = k < turned && !a.interleaved;
        offa[u] = half ? k * V : 2 * k * V;
        offb[u] = half ? a.rot / 2 + k * V : (2 * k + 1) * V;
        if (k < turned) {
            const int pos = a.positions[token];
            if (pos >= 0 && pos < a.max_pos) {
                const float *t = a.table + (long long)pos * a.rot + 2 * k * V;
#pragma unroll
                for (int i = 0; i < 2 * V; ++i) cs[u][i] = t[i];
            } else {   // no such position
#pragma unroll
                for (int i = 0; i < 2 * V; ++i) cs[u][i] = __builtin_nanf("");
            }
        }
        if (normed && mine[u]) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if (a.weight_f32) {
                    const float *g = static_cast<const float *>(a.weight[sec]);
                    w[u][i] = g[offa[u] + i];
                    w[u][V + i] = g[offb[u] + i];
                } else {
                    const T *g = static_cast<const T *>(a.weight[sec]);
                    w[u][i] = as_f32(g[offa[u] + i]);
                    w[u][V + i] = as_f32(g[offb[u] + i]);
                }
            }
        }
    }
    const int first = chunk * a.per_chunk, last = min(first + a.per_chunk, a.heads[sec]);
    for (int h0 = first; h0 < last; h0 += B) {
        Pack<T, V> pa[B][UPL], pb[B][UPL];
#pragma unroll
        for (int r = 0; r < B; ++r) {
            const T *row = x + (long long)min(h0 + r, last - 1) * a.xs[sec][1];
#pragma unroll
            for (int u = 0; u < UPL; ++u)
                if (mine[u]) {
                    pa[r][u].q = *reinterpret_cast<const typename Vec<T, V>::type *>(row + offa[u]);
                    pb[r][u].q = *reinterpret_cast<const typename Vec<T, V>::type *>(row + offb[u]);
                }
        }
#pragma unroll
        for (int r = 0; r < B; ++r) {
            if (h0 + r >= last) break;
            T *row = y + (long long)(h0 + r) * yh;
            float scale = 1.0f;
            if (normed) {
                float ss = 0.0f;
#pragma unroll
                for (int u = 0; u < UPL; ++u)
                    if (mine[u])
#pragma unroll
                        for (int i = 0; i < V; ++i) {
                            const float va = as_f32(pa[r][u].e[i]), vb = as_f32(pb[r][u].e[i]);
                            ss = fmaf(va, va, ss);
                            ss = fmaf(vb, vb, ss);
                        }
                scale = rsqrtf(group_sum<LPR>(ss) / (float)a.dim + a.eps);
            }
#pragma unroll
            for (int u = 0; u < UPL; ++u) {
                if (!mine[u]) continue;
                const bool turn = lane + u * LPR < turned;
                if (normed || turn) {
                    float f[2 * V];
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        f[i] = as_f32(pa[r][u].e[i]);
                        f[V + i] = as_f32(pb[r][u].e[i]);
                    }
                    if (normed)
#pragma unroll
                        for (int i = 0; i < 2 * V; ++i) f[i] = f[i] * scale * w[u][i];
                    if (turn) {
#pragma unroll
                        for (int p = 0; p < V; ++p) {
                            const float c = cs[u][2 * p], s = cs[u][2 * p + 1];
                            // a vector's neighbours, or the two vectors' values of the same index
                            const float n0 = f[2 * p], n1 = f[2 * p + 1], h0v = f[p], h1v = f[V + p];
                            const float va = a.interleaved ? n0 : h0v, vb = a.interleaved ? n1 : h1v;
                            const float ra = va * c - vb * s, rb = vb * c + va * s;
                            const int ia = 2 * p, ib = 2 * p + 1;
                            if (a.interleaved) {
                                put(ia < V ? pa[r][u].e[ia] : pb[r][u].e[ia - V], ra);
                                put(ib < V ? pa[r][u].e[ib] : pb[r][u].e[ib - V], rb);
                            } else {
                                put(pa[r][u].e[p], ra);
                                put(pb[r][u].e[p], rb);
                            }
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < V; ++i) {
                            put(pa[r][u].e[i], f[i]);
                            put(pb[r][u].e[i], f[V + i]);
                        }
                    }
                }
                typedef typename Vec<T, V>::type Q;
                Q *to_a = reinterpret_cast<Q *>(row + offa[u]), *to_b = reinterpret_cast<Q *>(row + offb[u]);
                if constexpr (PAST_L2) {
                    __builtin_nontemporal_store(pa[r][u].q, to_a);
                    __builtin_nontemporal_store(pb[r][u].q, to_b);
                } else {
                    *to_a = pa[r][u].q;
                    *to_b = pb[r][u].q;
                }
            }
        }
    }
}

template <typename T, int V, int LPR, int UPL>
hipError_t go(RopeArgs a, hipStream_t st) {
    const long long rows = a.heads[0] + a.heads[1] + a.heads[2];
    // heads a group: enough to read a table row and weights for several, few enough that the device is full (four
    // waves on each of its 1024 SIMDs): 8192 tokens of 40 heads of 128, eight heads 37.7 us, four 42.7
    const long long groups = 4096LL * (64 / LPR);
    a.per_chunk = 1;
    while (a.per_chunk < 8 && a.per_chunk * 2 * groups <= a.tokens * rows) a.per_chunk *= 2;
    // outputs that the L2s (eight of 4 MiB) will not keep for the next kernel are not kept in them: with
    // vectors of four, 8192 tokens of 40 heads of 128 in bf16 44.5 us for 46.9, 16384 tokens appended 28.5 for 34.2
    const bool past_l2 = a.tokens * rows * a.dim * (long long)sizeof(T) > (32LL << 20);
    a.all_chunks = 0;
    for (int s = 0; s < 3; ++s) a.all_chunks += a.chunks[s] = (a.heads[s] + a.per_chunk - 1) / a.per_chunk;
    a.div_chunks = fast_div((uint32_t)a.all_chunks);
    const long long ids = (long long)a.tokens * a.all_chunks;
    const long long blocks = (ids + kThreads / LPR - 1) / (kThreads / LPR);
    if (ids >= (1LL << 31) || blocks * kThreads >= (1LL << 32)) return hipErrorInvalidValue;   // past div_by, a launch
    if (past_l2) rope_kernel<T, V, LPR, UPL, true><<<(unsigned)blocks, kThreads, 0, st>>>(a);
    else rope_kernel<T, V, LPR, UPL, false><<<(unsigned)blocks, kThreads, 0, st>>>(a);
    return hipGetLastError();
}

template <typename T, int V> hipError_t pick(const RopeArgs &a, hipStream_t st) {
    const int units = a.dim / (2 * V);
    if constexpr (V > 1) {
        if (units <= 4) return go<T, V, 4, 1>(a, st);
        if (units <= 8) return go<T, V, 8, 1>(a, st);
        if (V == 8 || units <= 16) return go<T, V, 16, 1>(a, st);   // at most 128 / V units: dim <= 256
        if constexpr (V < 8) return go<T, V, 32, 1>(a, st);
    } else {
        if (units <= 32) return go<T, V, 32, 1>(a, st);
        if (units <= 64) return go<T, V, 64, 1>(a, st);
        return go<T, V, 64, 2>(a, st);
    }
}

__global__ __launch_bounds__(kThreads) void rope_table_kernel(ftcnn_rope_scaling sc, float2 *table) {
    const int half = sc.rot / 2;
    const long long i = (long long)blockIdx.x * kThreads + threadIdx.x;
    if (i >= (long long)sc.max_pos * half) return;
    const int pos = (int)(i / half), j = (int)(i % half);
    constexpr double two_pi = 6.283185307179586476925;
    const double base = sc.scaling == FTCNN_ROPE_BASE && sc.rot > 2
                            ? sc.base * pow(sc.factor, sc.rot / (sc.rot - 2.0)) : sc.base;
    double f = pow(base, -2.0 * j / sc.rot);
    if (sc.scaling == FTCNN_ROPE_LINEAR) {
        f /= sc.factor;
    } else if (sc.scaling == FTCNN_ROPE_PARTS) {
        const double turns = sc.original * f / two_pi;
        double keep = (turns - sc.low) / (sc.high - sc.low);
        keep = keep < 0.0 ? 0.0 : (keep > 1.0 ? 1.0 : keep);
        f *= keep + (1.0 - keep) / sc.factor;
    }
    double s, c;
    sincos(pos * f, &s, &c);
    table[i] = make_float2((float)(c * sc.amplitude), (float)(s * sc.amplitude));
}

}  // namespace

// Rows, their halves and the table start on whole vectors of `vec` values.
static bool rows_hold(const RopeArgs &a, int vec, int bytes) {
    auto off = [&](const void *p) { return reinterpret_cast<uintptr_t>(p) % bytes != 0; };
    if (a.dim % (2 * vec) || (a.positions && (a.rot % (2 * vec) || reinterpret_cast<uintptr_t>(a.table) % 16))) return false;
    for (int s = 0; s < 3; ++s) {
        if (!a.heads[s]) continue;
        if (off(a.x[s]) || off(a.y[s])) return false;
        for (int i = 0; i < 3; ++i)
            if ((i < 2 && a.xs[s][i] % vec) || a.ys[s][i] % vec) return false;
    }
    return true;
}

// The widest vectors that fit.  bf16, 8192 tokens of 40 heads: of 128 values, vectors of eight 37.7 us, of four 44.5; of
// 72, of four 35 us, single values 53.
hipError_t launch_rope(int dtype, const RopeArgs &a, hipStream_t st) {
    if (dtype == FTCNN_F32) return rows_hold(a, 4, 16) ? pick<float, 4>(a, st) : pick<float, 1>(a, st);
    if (rows_hold(a, 8, 16)) return pick<uint16_t, 8>(a, st);
    return rows_hold(a, 4, 8) ? pick<uint16_t, 4>(a, st) : pick<uint16_t, 1>(a, st);
}

hipError_t launch_rope_table(const ftcnn_rope_scaling &sc, float *table, hipStream_t st) {
    const long long n = (long long)sc.max_pos * (sc.rot / 2);
    if (n > (1LL << 32) - kThreads) return hipErrorInvalidValue;   // past a launch; 32 GB
    rope_table_kernel<<<(unsigned)((n + kThreads - 1) / kThreads), kThreads, 0, st>>>(
        sc, reinterpret_cast<float2 *>(table));
    return hipGetLastError();
}

}  // namespace ftcnn
