// Low-rank adapters of many requests beside a shared projection:
//
//   out_t = y_t + s_a B_a (A_a x_t),  a = ids[t],  A_a [rank][ch], B_a [m][rank],
//
// in two launches, each a matrix product with tiles of tokens: h = s A x, the channels split over a workgroup's
// waves, into the workspace, and out = y + B h.  A tile's tokens may have any adapters: its workgroups go over the different ones, each
// with the tokens that have it, the others' rows switched off.
#include <math.h>

#include <algorithm>

#include "low_rank.h"
#include "paged_attn.h"

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

// The tokens of one adapter that a wave multiplies together: whether there is a token `in` of the tile, and which.  Where there is
// none, one of the others, whose products go nowhere twice.
struct TileTokens {
    int t0, count;               // grouped: of the grouped tokens
    unsigned long long mine;     // not grouped: of the tile's tokens from t0 on, those with the adapter
    const int32_t *grouped;
    __device__ __forceinline__ bool has(int in) const { return grouped ? in < count : mine >> in & 1; }
    __device__ __forceinline__ int token(int in) const {
        return grouped ? grouped[t0 + min(in, count - 1)] : t0 + (mine >> in & 1 ? in : __builtin_ctzll(mine));
    }
};

// Calls f(adapter, its tokens) for the adapters of tile `tile`; adapter -1: tokens that have none.  By a whole wave.
// Grouped (few tokens of a tile have different adapters then): the tile is a record.  Else a tile is neighbouring tokens, and
// of their adapters those that fall to way `way` of `ways` are meant.
template <int TILE, bool GROUPED, typename F>
__device__ __forceinline__ void each_adapter(const LowRankArgs &a, int tile, int way, int ways, F f) {
    if constexpr (GROUPED) {
        if (tile >= *a.count) return;
        const int4 r = a.records[tile];
        f(__builtin_amdgcn_readfirstlane(r.x), TileTokens{r.y, r.z, 0, a.grouped});
    } else {
        const int lane = threadIdx.x & 63, t0 = tile * TILE, count = min(TILE, a.tokens - t0);
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
            if (k == way) f(adapter, TileTokens{t0, count, mine, nullptr});
        }
        if (none && way == 0) f(-1, TileTokens{t0, count, none, nullptr});
    }
}

constexpr int kGroup = 1024;   // threads of group_kernel

// The tokens of each adapter together, in tiles of `tile`: grouped[] has them one adapter's after the other's (those without one
// last), records[] (adapter, first of grouped, how many, 0) for each tile, *count how many.  One workgroup.  In which order an
// adapter's tokens come hangs on timing, and nothing on that: a row's products are its own.
__global__ __launch_bounds__(kGroup) void group_kernel(LowRankArgs a, int tile) {
    extern __shared__ __align__(16) int room[];
    const int bins = a.adapters + 1, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    int *tokens_of = room, *tiles_of = room + bins;   // counts, then where they begin
    __shared__ int sums[2][kGroup / 64];
    for (int i = tid; i < bins; i += kGroup) tokens_of[i] = 0;
    __syncthreads();
    auto bin = [&](int t) {
        const int id = a.ids[t];
        return (unsigned)id < (unsigned)a.adapters ? id : a.adapters;
    };
    // Adds the lanes to their bins' counts and returns what was there and in lower lanes: a wave whose tokens have one or two adapters (a
    // prompt's) with one addition for each.
    auto add = [&](int x, bool on) {
        int at = 0;
        unsigned long long left = __ballot(on);
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if (left) {
                const int first = __builtin_ctzll(left), theirs = __builtin_amdgcn_readlane(x, first);
                const unsigned long long same = __ballot(on && x == theirs) & left;
                int base = 0;
                if (lane == first) base = atomicAdd(&tokens_of[theirs], __popcll(same));
                base = __builtin_amdgcn_readlane(base, first);
                if (same >> lane & 1) at = base + __popcll(same & ((1ull << lane) - 1));
                left &= ~same;
            }
        if (left >> lane & 1) at = atomicAdd(&tokens_of[x], 1);
        return at;
    };
    for (int t0 = 0; t0 < a.tokens; t0 += kGroup) {
        const int t = t0 + tid;
        add(t < a.tokens ? bin(t) : 0, t < a.tokens);
    }
    __syncthreads();
    // where each bin's tokens and tiles begin: thread t has `run` bins from run * t on
    const int run = (bins + kGroup - 1) / kGroup, b0 = min(run * tid, bins), b1 = min(b0 + run, bins);
    int tokens = 0, tiles = 0;
    for (int i = b0; i < b1; ++i) {
        tokens += tokens_of[i];
        tiles += (tokens_of[i] + tile - 1) / tile;
    }
    int tokens_to = tokens, tiles_to = tiles;
#pragma unroll
    for (int x = 1; x < 64; x *= 2) {
        const int p = __shfl_up(tokens_to, x), q = __shfl_up(tiles_to, x);
        if (lane >= x) {
            tokens_to += p;
            tiles_to += q;
        }
    }
    if (lane == 63) {
        sums[0][w] = tokens_to;
        sums[1][w] = tiles_to;
    }
    __syncthreads();
    tokens_to -= tokens;
    tiles_to -= tiles;
    int total = 0;
    for (int i = 0; i < kGroup / 64; ++i) {
        if (i < w) {
            tokens_to += sums[0][i];
            tiles_to += sums[1][i];
        }
        total += sums[1][i];
    }
    for (int i = b0; i < b1; ++i) {
        const int n = tokens_of[i];
        tokens_of[i] = tokens_to;
        tiles_of[i] = tiles_to;
        tokens_to += n;
        tiles_to += (n + tile - 1) / tile;
    }
    __syncthreads();
    for (int i = tid; i < total; i += kGroup) {   // the bin of tile i: the last that begins at or before it, and is not empty
        int lo = 0, hi = bins;
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (tiles_of[mid] <= i) lo = mid;
            else hi = mid;
        }
        const int first = tokens_of[lo] + (i - tiles_of[lo]) * tile, end = lo + 1 < bins ? tokens_of[lo + 1] : a.tokens;
        a.records[i] = make_int4(lo < a.adapters ? lo : -1, first, min(tile, end - first), 0);
    }
    if (tid == 0) *a.count = total;
    __syncthreads();
    for (int t0 = 0; t0 < a.tokens; t0 += kGroup) {
        const int t = t0 + tid, at = add(t < a.tokens ? bin(t) : 0, t < a.tokens);
        if (t < a.tokens) a.grouped[at] = t;
    }
}

__device__ __forceinline__ int used_rank(const LowRankArgs &a, int adapter) {
    return a.ranks ? min(max(a.ranks[adapter], 0), a.rank) : a.rank;
}

constexpr int kShrinkWaves = 8;

// The products of a tile's tokens with 16 NB rows of their adapter's A.  A workgroup's waves share its channels, each keeps AHEAD
// chunks of every row on their way while it multiplies as many, and their sums are added in LDS.  Rows of tokens that have another adapter,
// and those past the rank, are read as ones that are there: their products go nowhere.
template <typename T, int MT, int NB, bool GROUPED>
__global__ __launch_bounds__(64 * kShrinkWaves) void shrink_kernel(LowRankArgs a) {
    using C = Chunk<T>;
    constexpr int W = kShrinkWaves, TILE = 16 * MT, RANK = 16 * NB, AHEAD = MT + NB <= 3 ? 4 : (MT + NB <= 6 ? 2 : 1);
    extern __shared__ __align__(16) float sums[];   // [W][TILE][RANK]
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n16 = lane & 15, h = lane >> 4;
    const unsigned x1 = div_by(blockIdx.x, a.div_groups), x2 = div_by(x1, a.div_splits), x3 = div_by(x2, a.div_ways);
    const int r0 = (int)(blockIdx.x - x1 * a.groups) * RANK, split = (int)(x1 - x2 * a.splits);
    const int way = (int)(x2 - x3 * a.ways);
    // This wave's channels: every (splits * W)-th block of 256 bytes of a row, so that the waves, whose rows often lie a power of
    // two apart, are at different memory channels; AHEAD chunks of 64 bytes at a time, the last block perhaps in part.
    const int chunks = (a.ch + C::VALUES - 1) / C::VALUES, whole = a.ch / C::VALUES, part = split * W + w, parts = a.splits * W;
    const int blocks = max((whole / 4 - part + parts - 1) / parts, 0), groups = blocks * (4 / AHEAD);
    const auto chunk_of = [&](int g) { return (part + g / (4 / AHEAD) * parts) * 4 + g % (4 / AHEAD) * AHEAD; };
    each_adapter<TILE, GROUPED>(a, (int)x3, way, a.ways, [&](int adapter, const TileTokens &tokens) __attribute__((always_inline)) {
        if (adapter < 0) return;
        const int rank = used_rank(a, adapter);
        const T *xr[MT], *ar[NB];
#pragma unroll
        for (int i = 0; i < MT; ++i)
            xr[i] = static_cast<const T *>(a.x) + tokens.token(16 * i + n16) * a.xs + h * C::EU;
#pragma unroll
        for (int j = 0; j < NB; ++j)
            ar[j] = static_cast<const T *>(a.a) + adapter * a.as[0] + min(r0 + 16 * j + n16, a.rank - 1) * a.as[1] + h * C::EU;
        f32x4 acc[MT][NB];
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        struct Stage {
            uint4 x[AHEAD][MT], a[AHEAD][NB];
        } s0, s1;
        auto load = [&](Stage &s, int c) __attribute__((always_inline)) {
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const int at = (c + k) * C::VALUES;
#pragma unroll
                for (int i = 0; i < MT; ++i) s.x[k][i] = *reinterpret_cast<const uint4 *>(xr[i] + at);
#pragma unroll
                for (int j = 0; j < NB; ++j) s.a[k][j] = *reinterpret_cast<const uint4 *>(ar[j] + at);
            }
        };
        auto multiply = [&](const Stage &s) __attribute__((always_inline)) {
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int j = 0; j < NB; ++j) acc[i][j] = product<T>(s.x[k][i], s.a[k][j], acc[i][j]);
        };
        // (no loads under conditions in the loop: the wait for one stage would be for both)
        if (groups > 0) {
            load(s0, chunk_of(0));
            int g = 0;
            for (; g + 2 < groups; g += 2) {
                load(s1, chunk_of(g + 1));
                __builtin_amdgcn_sched_barrier(0);
                multiply(s0);
                load(s0, chunk_of(g + 2));
                __builtin_amdgcn_sched_barrier(0);
                multiply(s1);
            }
            if (g + 1 < groups) {
                load(s1, chunk_of(g + 1));
                multiply(s0);
                multiply(s1);
            } else {
                multiply(s0);
            }
        }
        // the row's last chunks, less than a block: one for each wave of the last range
        for (int c = whole / 4 * 4 + w; c < chunks && split == a.splits - 1; c += W) {
            const int at = c * C::VALUES;
            const bool on = at + h * C::EU < a.ch;
            uint4 xf[MT];
#pragma unroll
            for (int i = 0; i < MT; ++i) xf[i] = on ? *reinterpret_cast<const uint4 *>(xr[i] + at) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                const uint4 af = on ? *reinterpret_cast<const uint4 *>(ar[j] + at) : make_uint4(0, 0, 0, 0);
#pragma unroll
                for (int i = 0; i < MT; ++i) acc[i][j] = product<T>(xf[i], af, acc[i][j]);
            }
        }
        // rows 4 h + e of tokens, column n16 of the rank
        __syncthreads();   // the adapter before this one
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) sums[(w * TILE + 16 * i + 4 * h + e) * RANK + 16 * j + n16] = acc[i][j][e];
        __syncthreads();
        const float s = a.scales ? a.scales[adapter] : 1.0f;
        for (int i = threadIdx.x; i < TILE * RANK; i += 64 * W) {
            const int t = i / RANK, r = r0 + i % RANK;
            if (!tokens.has(t) || r >= a.rank) continue;
            float v = sums[i];
#pragma unroll
            for (int k = 1; k < W; ++k) v += sums[k * TILE * RANK + i];
            a.low[((long long)split * a.tokens + tokens.token(t)) * a.rank + r] = r < rank ? s * v : 0.0f;
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

template <typename T> union Unit {
    uint4 q;
    T e[16 / sizeof(T)];
};
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
// outputs of a token.  A wave has its tile's h in registers and goes over some outputs, 64 at a time, those of y and B on their
// way while the ones before are multiplied.
//
// bf16: h is the sum of two bf16 values (an error of 2^-17 of it; rounded to one, its products would be off by as
// much as the outputs' own rounding).
template <typename T, int MT, int RC, bool GROUPED>
__global__ __launch_bounds__(256) void expand_kernel(LowRankArgs a) {
    using C = Chunk<T>;
    constexpr int EU = C::EU, TILE = 16 * MT, PLANES = sizeof(T) == 2 ? 2 : 1, SZ = (int)sizeof(T);
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n16 = lane & 15, h = lane >> 4;
    const unsigned x1 = div_by(blockIdx.x, a.div_spans), x2 = div_by(x1, a.div_expand_ways);
    const int way = (int)(x1 - x2 * a.expand_ways);
    // a workgroup's waves have `together` tiles (one or four), which share the loads of B, and one or four spans of outputs
    const long long tile = (long long)x2 * a.together + (a.together > 1 ? w : 0);
    const long long span = a.together > 1 ? blockIdx.x - x1 * a.div_spans.d : (long long)(blockIdx.x - x1 * a.div_spans.d) * 4 + w;
    if (tile >= a.tiles) return;
    const int m0 = (int)min(span * a.columns, (long long)a.m), m1 = (int)min((span + 1) * a.columns, (long long)a.m);
    if (m0 >= m1) return;
    each_adapter<TILE, GROUPED>(a, (int)tile, way, a.expand_ways, [&](int adapter, const TileTokens &tokens) __attribute__((always_inline)) {
        if (adapter < 0) {   // no adapter: as they are
            for (int i = 0; a.out != a.y && i < TILE; ++i) {
                if (!tokens.has(i)) continue;
                const long long t = tokens.token(i);
                const T *y = static_cast<const T *>(a.y) + t * a.ys;
                T *out = static_cast<T *>(a.out) + t * a.os;
                for (int c = m0 + EU * lane; c < m1; c += EU * 64)
                    *reinterpret_cast<uint4 *>(out + c) = *reinterpret_cast<const uint4 *>(y + c);
            }
            return;
        }
        const int rank = used_rank(a, adapter);
        const T *bt = static_cast<const T *>(a.b) + adapter * a.bs[0];
        // workgroups begin at different places of their span: rows of y often lie a power of two apart, and 64 of its
        // columns in all rows at one memory channel
        const int steps = (m1 - m0 + 63) / 64, turn = (int)(x2 % (unsigned)steps);
        auto place = [&](int i) __attribute__((always_inline)) { return m0 + 64 * (i + turn < steps ? i + turn : i + turn - steps); };
        bool on[MT];
        const T *yt[MT];
        T *ot[MT];
        uint4 low[MT][RC][PLANES];   // (of other tokens any values: their products go nowhere)
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            on[i] = tokens.has(16 * i + n16);
            const long long t = tokens.token(16 * i + n16);
            yt[i] = static_cast<const T *>(a.y) + t * a.ys + 16 * h;
            ot[i] = static_cast<T *>(a.out) + t * a.os + 16 * h;
#pragma unroll
            for (int c = 0; c < RC; ++c) {
                const int k = c * C::VALUES + h * EU;
                float v[EU];
#pragma unroll
                for (int e = 0; e < EU; ++e) v[e] = 0.0f;
                if (k < a.rank)
                    for (int s = 0; s < a.splits; ++s) {
                        const float4 *from = reinterpret_cast<const float4 *>(a.low + (s * (long long)a.tokens + t) * a.rank + k);
#pragma unroll
                        for (int e = 0; e < EU; e += 4) {
                            const float4 f = from[e / 4];
                            v[e] += f.x;
                            v[e + 1] += f.y;
                            v[e + 2] += f.z;
                            v[e + 3] += f.w;
                        }
                    }
                Unit<T> hi, lo;
#pragma unroll
                for (int e = 0; e < EU; ++e) {
                    narrow(hi.e[e], v[e]);
                    const float top = widen(hi.e[e]);
                    narrow(lo.e[e], fabsf(top) < INFINITY ? v[e] - top : 0.0f);   // (of an infinity or NaN there is no rest)
                }
                low[i][c][0] = hi.q;
                if constexpr (PLANES == 2) low[i][c][PLANES - 1] = lo.q;
            }
        }
        struct Stage {
            Row16<T> y[MT];
            uint4 b[RC][4];
        };
        auto load = [&](Stage &s, int i) __attribute__((always_inline)) {
            const int m = place(i);
#pragma unroll
            for (int c = 0; c < RC; ++c)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int row = m + 16 * (n16 >> 2) + 4 * q + (n16 & 3), k = c * C::VALUES + h * EU;
                    // rows past the last: that one, for nobody; past the rank: zero, as h is
                    s.b[c][q] = *reinterpret_cast<const uint4 *>(bt + min(row, m1 - 1) * a.bs[1] + min(k, a.rank - EU));
                }
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int u = 0; u < SZ; ++u)
                    s.y[t].q[u] = *reinterpret_cast<const uint4 *>(yt[t] + min(m + u * EU, m1 - EU - 16 * h));
        };
        auto multiply = [&](Stage &s, int i) __attribute__((always_inline)) {
            const int m = place(i);
            f32x4 acc[4][MT];
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int t = 0; t < MT; ++t) acc[q][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int c = 0; c < RC; ++c) {
                const int k = c * C::VALUES + h * EU;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const uint4 b = rank < RC * C::VALUES ? within_rank<T>(s.b[c][q], k, rank) : s.b[c][q];
#pragma unroll
                    for (int t = 0; t < MT; ++t)
#pragma unroll
                        for (int p = 0; p < PLANES; ++p) acc[q][t] = product<T>(b, low[t][c][p], acc[q][t]);
                }
            }
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                Row16<T> v;
#pragma unroll
                for (int e = 0; e < 16; ++e) narrow(v.e[e], widen(s.y[t].e[e]) + acc[e / 4][t][e % 4]);
#pragma unroll
                for (int u = 0; u < SZ; ++u)
                    if (on[t] && m + 16 * h + u * EU < m1) *reinterpret_cast<uint4 *>(ot[t] + m + u * EU) = v.q[u];
            }
        };
        Stage s0, s1;
        load(s0, 0);
        int i = 0;
        for (; i + 2 < steps; i += 2) {
            load(s1, i + 1);
            __builtin_amdgcn_sched_barrier(0);
            multiply(s0, i);
            load(s0, i + 2);
            __builtin_amdgcn_sched_barrier(0);
            multiply(s1, i + 1);
        }
        if (i + 1 < steps) {
            load(s1, i + 1);
            multiply(s0, i);
            multiply(s1, i + 1);
        } else {
            multiply(s0, i);
        }
    });
}

template <typename T, int MT, int NB, bool GROUPED> hipError_t shrink_go(const LowRankPlan &pl, const LowRankArgs &a, hipStream_t st) {
    constexpr int LDS = kShrinkWaves * 16 * MT * 16 * NB * (int)sizeof(float);
    auto kernel = shrink_kernel<T, MT, NB, GROUPED>;
    if constexpr (LDS > 65536) {
        static std::atomic<uint64_t> raised{0};   // devices whose limit is raised for this kernel
        const hipError_t err = raise_lds_limit(reinterpret_cast<const void *>(kernel), LDS, raised);
        if (err != hipSuccess) return err;
    }
    kernel<<<(unsigned)pl.tiles * pl.ways * pl.splits * pl.groups, 64 * kShrinkWaves, LDS, st>>>(a);
    return hipGetLastError();
}
template <typename T, int MT, bool GROUPED> hipError_t go(const LowRankPlan &pl, const LowRankArgs &a, hipStream_t st) {
    const hipError_t err = pl.blocks == 1   ? shrink_go<T, MT, 1, GROUPED>(pl, a, st)
                           : pl.blocks == 2 ? shrink_go<T, MT, 2, GROUPED>(pl, a, st)
                           : pl.blocks == 4 ? shrink_go<T, MT, 4, GROUPED>(pl, a, st)
                                            : shrink_go<T, MT, 8, GROUPED>(pl, a, st);
    if (err != hipSuccess) return err;
    const unsigned blocks = (unsigned)((pl.tiles + pl.together - 1) / pl.together) * pl.expand_ways * pl.spans;
    constexpr int V = Chunk<T>::VALUES;
    if (a.rank <= V) expand_kernel<T, MT, 1, GROUPED><<<blocks, 256, 0, st>>>(a);
    else if (a.rank <= 2 * V) expand_kernel<T, MT, 2, GROUPED><<<blocks, 256, 0, st>>>(a);
    else if (a.rank <= 4 * V) expand_kernel<T, MT, 4, GROUPED><<<blocks, 256, 0, st>>>(a);
    else if constexpr (sizeof(T) == 4) expand_kernel<T, MT, 8, GROUPED><<<blocks, 256, 0, st>>>(a);
    return hipGetLastError();
}
template <typename T> hipError_t pick(const LowRankPlan &pl, const LowRankArgs &a, hipStream_t st) {
    if (pl.grouped) return pl.tile == 16 ? go<T, 1, true>(pl, a, st) : go<T, 2, true>(pl, a, st);
    return pl.tile == 16 ? go<T, 1, false>(pl, a, st) : go<T, 2, false>(pl, a, st);
}

// Bins of group_kernel, two counts each, that LDS holds without more of it being asked for.
constexpr int kMaxBins = 8000;

}  // namespace

LowRankPlan low_rank_plan(const ftcnn_low_rank_desc &d) {
    LowRankPlan p{};
    if (d.tokens == 0) return p;
    p.grouped = d.tokens >= 512 && d.adapters > 1 && d.adapters < kMaxBins;
    // two tiles of 16 together where they fill the device and adapters have as many tokens
    p.tile = d.tokens >= 32 * kComputeUnits / 2 && d.tokens / d.adapters >= 32 ? 32 : 16;
    p.tiles = (d.tokens + p.tile - 1) / p.tile + (p.grouped ? std::min(d.adapters, d.tokens) : 0);
    const long long most = p.grouped ? 1 : std::max(1, std::min(p.tile, d.adapters));
    auto share = [&](long long want, long long have) { return (int)std::max(1LL, std::min(most, want / std::max(1LL, have))); };
    // rows of A together where tiles fill the device, apart where they do not
    const int rows = (d.rank + 15) / 16;
    p.blocks = rows > 4 ? 8 : (rows > 2 ? 4 : rows);
    while (p.blocks > 1 && (long long)p.tiles * ((rows + p.blocks - 1) / p.blocks) < kComputeUnits) p.blocks /= 2;
    p.groups = (rows + p.blocks - 1) / p.blocks;
    p.ways = share(2 * kComputeUnits, (long long)p.tiles * p.groups);
    // ranges of channels where there are too few workgroups still: four chunks of 64 bytes a wave at least
    const long long chunks = ((long long)d.ch * (d.dtype == FTCNN_F32 ? 4 : 2) + 63) / 64;
    p.splits = (int)std::max(1LL, std::min(chunks / (4 * kShrinkWaves), 2LL * kComputeUnits / ((long long)p.tiles * p.groups * p.ways)));
    // outputs of a wave: as many as leave eight waves to a compute unit
    const long long blocks = (d.m + 63) / 64;
    p.expand_ways = share(8 * kComputeUnits, p.tiles * ((blocks + 3) / 4));
    const long long waves = p.tiles * p.expand_ways * blocks;
    const long long each = std::max(1LL, std::min(blocks, waves / (8LL * kComputeUnits)));
    p.together = p.tiles >= 64 ? 4 : 1;
    const long long of_group = each * (4 / p.together);
    p.columns = (int)(64 * each);
    p.spans = (int)((blocks + of_group - 1) / of_group);
    auto up = [](size_t x) { return (x + 255) & ~size_t(255); };
    p.records = up((size_t)p.splits * d.tokens * d.rank * sizeof(float));
    p.bytes = p.records;
    if (p.grouped) {
        p.order = p.records + up((size_t)p.tiles * sizeof(int4));
        p.count = p.order + up((size_t)d.tokens * sizeof(int32_t));
        p.bytes = p.count + 256;
    }
    return p;
}

hipError_t launch_low_rank(int dtype, const LowRankPlan &pl, const LowRankArgs &a, hipStream_t st) {
    if (pl.grouped) {
        group_kernel<<<1, kGroup, 2 * (a.adapters + 1) * sizeof(int), st>>>(a, pl.tile);
        const hipError_t err = hipGetLastError();
        if (err != hipSuccess) return err;
    }
    return dtype == FTCNN_F32 ? pick<float>(pl, a, st) : pick<uint16_t>(pl, a, st);
}

}  // namespace ftcnn
