// Low-rank adapters of many requests beside a shared projection:
//
//   out_t = y_t + s_a B_a (A_a x_t),  a = ids[t],  A_a [rank][ch], B_a [m][rank],
//
// in two launches, each a matrix product with tiles of tokens: h = s A x, the channels split over a workgroup's
// waves, into the workspace, and out = y + B h.  A tile's tokens may have any adapters: its workgroups go over the
// different ones, each with the tokens that have it, the others' rows switched off.  Where that reads much, a launch before
// them groups the tokens by adapter, and a tile has one.  Small calls have one launch for both products.
//
// Few tokens: latency bounds every launch: 9 us for one token in one launch (4096 channels, 6144 outputs, rank 16, bf16; at a
// copy's rate its 0.4 MB take 0.07), 6.8 and 8.4 for 64 tokens of 48 adapters of rank 32 (4.5 us for their bytes, if each
// came once).  Many: x, y and the output at memory's rate.  8192 tokens of six adapters, 4096 channels and outputs, rank 64:
// 5, 31 and 43 us, of which a copy's rate would take 40 in all; the last also asks the first-level cache for B, 0.5 MB, for
// every tile of 32 tokens.
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

// Calls f(adapter, its tokens) for the adapters of tile `tile` of neighbouring tokens, of these those that fall to way `way` of
// `ways`; adapter -1: tokens that have none.  By a whole wave.
template <int TILE, typename F>
__device__ __forceinline__ void each_adapter(const LowRankArgs &a, int tile, int way, int ways, F f) {
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

constexpr int kGroup = 1024, kPart = 2 * kGroup;   // threads of group_kernel; tokens of a workgroup of it

// The tokens of each adapter together, in tiles of `tile`, of every part of kPart tokens for itself: grouped[] has them one
// adapter's after the other's (those without one last), records[] (adapter, first of grouped, how many, 0) for each tile, slots
// of them a part, counts[] how many.  A workgroup a part.  In which order an adapter's tokens come hangs on timing, and nothing
// on that: a row's products are its own.
__global__ __launch_bounds__(kGroup) void group_kernel(LowRankArgs a, int tile) {
    extern __shared__ __align__(16) int room[];
    const int bins = a.adapters + 1, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int t0 = blockIdx.x * kPart, end = min(t0 + kPart, a.tokens);
    int *tokens_of = room, *tiles_of = room + bins;   // counts, then where they begin
    __shared__ int sums[2][kGroup / 64];
    int x[2], at[2];   // this lane's tokens: the bin, the place in it
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int t = t0 + i * kGroup + tid, id = t < end ? a.ids[t] : -1;
        x[i] = (unsigned)id < (unsigned)a.adapters ? id : a.adapters;
    }
    for (int i = tid; i < bins; i += kGroup) tokens_of[i] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const bool on = t0 + i * kGroup + tid < end;
        // a wave whose tokens have one adapter (a prompt's), or many of them the first one's, does one addition for those
        const unsigned long long left = __ballot(on);
        if (left == 0) continue;
        const int theirs = __builtin_amdgcn_readlane(x[i], __builtin_ctzll(left));
        const unsigned long long same = __ballot(on && x[i] == theirs);
        int base = 0;
        if (lane == 0) base = atomicAdd(&tokens_of[theirs], __popcll(same));
        if (on && x[i] != theirs) at[i] = atomicAdd(&tokens_of[x[i]], 1);
        base = __builtin_amdgcn_readfirstlane(base);
        if (on && x[i] == theirs) at[i] = base + __popcll(same & ((1ull << lane) - 1));
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
    for (int y = 1; y < 64; y *= 2) {
        const int p = __shfl_up(tokens_to, y), q = __shfl_up(tiles_to, y);
        if (lane >= y) {
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
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int t = t0 + i * kGroup + tid;
        if (t < end) a.grouped[t0 + tokens_of[x[i]] + at[i]] = t;
    }
    if (tid == 0) a.counts[blockIdx.x] = total;
    for (int i = tid; i < total; i += kGroup) {   // the bin of tile i: the last that begins at or before it
        int lo = 0, hi = bins;
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (tiles_of[mid] <= i) lo = mid;
            else hi = mid;
        }
        const int first = tokens_of[lo] + (i - tiles_of[lo]) * tile, next = lo + 1 < bins ? tokens_of[lo + 1] : end - t0;
        a.records[(long long)blockIdx.x * a.slots + i] = make_int4(lo < a.adapters ? lo : -1, t0 + first, min(tile, next - first), 0);
    }
}

__device__ __forceinline__ int used_rank(const LowRankArgs &a, int adapter) {
    return a.ranks ? min(max(a.ranks[adapter], 0), a.rank) : a.rank;
}

constexpr int kShrinkWaves = 8;

// The products of a tile's tokens with 16 NB rows of their adapter's A.  A workgroup's waves share its channels, each keeps AHEAD
// chunks of every row on their way while it multiplies as many, and their sums are added in LDS.  Rows of tokens that have another adapter,
// and those past the rank, are read as ones that are there: their products go nowhere.
template <typename T, int MT, int NB> struct Shrink {
    static constexpr int W = kShrinkWaves, TILE = 16 * MT, RANK = 16 * NB, AHEAD = MT + NB <= 3 ? 4 : (MT + NB <= 6 ? 2 : 1);
    static constexpr int SUMS = W * TILE * RANK;   // floats in LDS, [W][TILE][RANK]
    // Of rows r0 on and range `split` of the channels, every wave's part into `sums`, by a whole workgroup.
    __device__ static __forceinline__ void parts(const LowRankArgs &a, int adapter, const TileTokens &tokens, int r0, int split, float *sums);
    __device__ static __forceinline__ float sum(const float *sums, int i) {   // of value i
        float v = sums[i];
#pragma unroll
        for (int k = 1; k < W; ++k) v += sums[k * TILE * RANK + i];
        return v;
    }
};
template <typename T, int MT, int NB>
__device__ __forceinline__ void Shrink<T, MT, NB>::parts(const LowRankArgs &a, int adapter, const TileTokens &tokens, int r0, int split,
                                                         float *sums) {
    using C = Chunk<T>;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n16 = lane & 15, h = lane >> 4;
    // This wave's channels: every (splits * W)-th block of 256 bytes of a row, so that the waves, whose rows often lie a power of
    // two apart, are at different memory channels; AHEAD chunks of 64 bytes at a time, the last block perhaps in part.
    const int chunks = (a.ch + C::VALUES - 1) / C::VALUES, whole = a.ch / C::VALUES, part = split * W + w, all = a.splits * W;
    const int blocks = max((whole / 4 - part + all - 1) / all, 0), groups = blocks * (4 / AHEAD);
    const auto chunk_of = [&](int g) { return (part + g / (4 / AHEAD) * all) * 4 + g % (4 / AHEAD) * AHEAD; };
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
}

template <typename T, int MT, int NB>
__global__ __launch_bounds__(64 * kShrinkWaves) void shrink_kernel(LowRankArgs a) {
    using S = Shrink<T, MT, NB>;
    extern __shared__ __align__(16) float sums[];
    const unsigned x1 = div_by(blockIdx.x, a.div_groups), x2 = div_by(x1, a.div_splits), x3 = div_by(x2, a.div_ways);
    const int r0 = (int)(blockIdx.x - x1 * a.groups) * S::RANK, split = (int)(x1 - x2 * a.splits);
    const int way = (int)(x2 - x3 * a.ways);
    each_adapter<S::TILE>(a, (int)x3, way, a.ways, [&](int adapter, const TileTokens &tokens) __attribute__((always_inline)) {
        if (adapter < 0) return;
        const int rank = used_rank(a, adapter);
        S::parts(a, adapter, tokens, r0, split, sums);
        const float s = a.scales ? a.scales[adapter] : 1.0f;
        for (int i = threadIdx.x; i < S::TILE * S::RANK; i += 64 * S::W) {
            const int t = i / S::RANK, r = r0 + i % S::RANK;
            if (!tokens.has(t) || r >= a.rank) continue;
            a.low[((long long)split * a.tokens + tokens.token(t)) * a.rank + r] = r < rank ? s * S::sum(sums, i) : 0.0f;
        }
    });
}

// The same for grouped tokens, of which there are many: rows of tokens and of A come into LDS in pieces of 256 bytes, whole lines of
// neighbouring lanes (a load in the order of the operands touches sixteen lines for each 256 bytes of it, and the first-level cache
// looks one up a cycle), DEPTH - 1 pieces ahead, and every wave multiplies 64 bytes of each row of a piece.
template <typename T, int MT, int NB> struct Ring {
    static constexpr int ROWS = 16 * (MT + NB), PIECE = 256, STAGE = ROWS * PIECE;
    static constexpr int LOADS = ROWS / 16;                                  // of a wave and stage, four rows each
    static constexpr int DEPTH = 81920 / STAGE < 8 ? 81920 / STAGE : 8, LDS = DEPTH * STAGE;   // two workgroups to a compute unit
    static_assert(DEPTH >= 2 && (DEPTH - 2) * LOADS < 64 && 4 * 16 * MT * 16 * NB * 4 <= LDS, "the waits count to 63; the sums fit");
};
template <int N> __device__ __forceinline__ void wait_all_but() {   // all but the last N loads of this wave have landed
    __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | (N >> 4) << 14);
    asm volatile("" ::: "memory");
}

template <typename T, int MT, int NB>
__global__ __launch_bounds__(256) void shrink_ring_kernel(LowRankArgs a) {
    using C = Chunk<T>;
    using R = Ring<T, MT, NB>;
    constexpr int EU = C::EU, TILE = 16 * MT, RANK = 16 * NB, PER = 16 * EU;   // values of a piece of a row
    extern __shared__ __align__(1024) unsigned char ring[];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n16 = lane & 15, h = lane >> 4;
    typedef __attribute__((address_space(3))) unsigned char lds_byte;
    const unsigned ring_at = (unsigned)(uintptr_t)(lds_byte *)ring;
    const unsigned x1 = div_by(blockIdx.x, a.div_groups), x2 = div_by(x1, a.div_splits);
    const int r0 = (int)(blockIdx.x - x1 * a.groups) * RANK, split = (int)(x1 - x2 * a.splits);
    const int of = (int)div_by(x2, a.div_slots);
    if ((int)x2 - of * a.slots >= a.counts[of]) return;
    const int4 record = a.records[x2];
    const int adapter = __builtin_amdgcn_readfirstlane(record.x);
    if (adapter < 0) return;
    const TileTokens tokens{record.y, record.z, 0, a.grouped};
    const int rank = used_rank(a, adapter);
    // this workgroup's pieces of every row
    const int pieces = (a.ch + PER - 1) / PER, each = (int)div_by(pieces, a.div_splits), more = pieces - each * a.splits;
    const int p0 = each * split + min(split, more), count = each + (split < more ? 1 : 0);
    // this wave's loads: four rows each, tokens first, then A; the unit of a row that belongs at this lane's place.  Rows of no token,
    // and those past the rank, are others' that are there: their products go nowhere.
    const char *from[R::LOADS];
    int unit[R::LOADS];
#pragma unroll
    for (int i = 0; i < R::LOADS; ++i) {
        const int row = 4 * (4 * i + w) + h;   // 4 i + w: of 4 (MT + NB) loads
        unit[i] = n16 ^ (row & 15);
        const T *at = row < TILE ? static_cast<const T *>(a.x) + tokens.token(row) * a.xs
                                 : static_cast<const T *>(a.a) + adapter * a.as[0] + min(r0 + row - TILE, a.rank - 1) * a.as[1];
        from[i] = reinterpret_cast<const char *>(at + (long long)p0 * PER) + unit[i] * 16;
    }
    auto issue = [&](int t) __attribute__((always_inline)) {   // piece p0 + t
        const unsigned to = ring_at + t % R::DEPTH * R::STAGE + w * 1024;
        const int left = a.ch - (p0 + t) * PER;   // values of the row from this piece on
        if (left >= PER) {
#pragma unroll
            for (int i = 0; i < R::LOADS; ++i) load_to_lds(from[i] + (long long)t * 256, to + i * 4096);
        } else {
#pragma unroll
            for (int i = 0; i < R::LOADS; ++i)
                if (unit[i] * EU < left) load_to_lds(from[i] + (long long)t * 256, to + i * 4096);
        }
    };
    f32x4 acc[MT][NB];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    wait_loads();   // what came before is not counted below
    for (int t = 0; t < R::DEPTH - 1 && t < count; ++t) issue(t);
    for (int t = 0; t < count; ++t) {
        if (t + R::DEPTH - 1 <= count) wait_all_but<(R::DEPTH - 2) * R::LOADS>();
        else wait_loads();
        tile_barrier();   // piece t has landed, and nobody reads piece t - 1 any more
        if (t + R::DEPTH - 1 < count) issue(t + R::DEPTH - 1);
        const unsigned char *at = ring + t % R::DEPTH * R::STAGE + (((4 * w + h) ^ n16) << 4) + n16 * 256;
        uint4 xf[MT], af[NB];
#pragma unroll
        for (int i = 0; i < MT; ++i) xf[i] = *reinterpret_cast<const uint4 *>(at + 16 * i * 256);
#pragma unroll
        for (int j = 0; j < NB; ++j) af[j] = *reinterpret_cast<const uint4 *>(at + (TILE + 16 * j) * 256);
        if ((p0 + t + 1) * PER > a.ch && (p0 + t) * PER + (4 * w + h) * EU >= a.ch) {   // past the channels: LDS holds anything
#pragma unroll
            for (int i = 0; i < MT; ++i) xf[i] = make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int j = 0; j < NB; ++j) af[j] = make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j) acc[i][j] = product<T>(xf[i], af[j], acc[i][j]);
    }
    __syncthreads();
    float *sums = reinterpret_cast<float *>(ring);   // [4][TILE][RANK]
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) sums[(w * TILE + 16 * i + 4 * h + e) * RANK + 16 * j + n16] = acc[i][j][e];
    __syncthreads();
    const float s = a.scales ? a.scales[adapter] : 1.0f;
    for (int i = threadIdx.x; i < TILE * RANK; i += 256) {
        const int t = i / RANK, r = r0 + i % RANK;
        if (!tokens.has(t) || r >= a.rank) continue;
        float v = sums[i];
#pragma unroll
        for (int k = 1; k < 4; ++k) v += sums[k * TILE * RANK + i];
        a.low[((long long)split * a.tokens + tokens.token(t)) * a.rank + r] = r < rank ? s * v : 0.0f;
    }
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
__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(uint16_t v) { return bf16_bits_to_f32(v); }
__device__ __forceinline__ void narrow(float &d, float v) { d = v; }
__device__ __forceinline__ void narrow(uint16_t &d, float v) { d = f32_to_bf16_rne(v); }

// The product is O^T = B H^T: a lane has a token, and of each of four blocks of 16 outputs the rows 4 h + e.
// Row 4 g + e of block q is output 16 g + 4 q + e, so that a lane's 16 values are neighbours and four lanes hold 64
// outputs of a token.  A wave has its tile's h in registers and goes over some outputs, 64 at a time, those of y and B on their
// way while the ones before are multiplied.  The products go through LDS, which each wave has for itself, so that y and the
// output are read and written in whole lines (see Ring).
//
// bf16: h is the sum of two bf16 values (an error of 2^-17 of it; rounded to one, its products would be off by as
// much as the outputs' own rounding).
constexpr float kLargest = 0x1.fep127f;   // of bf16
__device__ __forceinline__ int output_row(int n16, int q) { return 16 * (n16 >> 2) + 4 * q + (n16 & 3); }

// h of a tile's tokens, as operands: unit c * 4 + h of token 16 i + n16.  (Of tokens that are none, of others: their products go
// nowhere.)
template <typename T, int MT, int RC> struct Low {
    static constexpr int EU = 16 / sizeof(T), PLANES = sizeof(T) == 2 ? 2 : 1;
    uint4 low[MT][RC][PLANES];
    // acc[q] += unit (c, q) of B times these
    __device__ __forceinline__ void multiply(f32x4 (&acc)[4][MT], int c, int q, uint4 b) const {
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int p = 0; p < PLANES; ++p) acc[q][t] = product<T>(b, low[t][c][p], acc[q][t]);
    }
    // row(i): h of the tile's token i, of `splits` ranges of channels, tokens * rank values apart
    template <typename F> __device__ __forceinline__ void load(const LowRankArgs &a, int splits, F row) {
        const int n16 = threadIdx.x & 15, h = (threadIdx.x & 63) >> 4;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const float *of = row(16 * i + n16);
#pragma unroll
            for (int c = 0; c < RC; ++c) {
                const int k = (4 * c + h) * EU;
                float v[EU];
#pragma unroll
                for (int e = 0; e < EU; ++e) v[e] = 0.0f;
                if (k < a.rank) {
                    const float *from = of + k;
                    const long long step = (long long)a.tokens * a.rank;
                    auto add = [&](float4 f, int e) __attribute__((always_inline)) {
                        v[e] += f.x;
                        v[e + 1] += f.y;
                        v[e + 2] += f.z;
                        v[e + 3] += f.w;
                    };
                    if (splits == 1) {
#pragma unroll
                        for (int e = 0; e < EU; e += 4) add(reinterpret_cast<const float4 *>(from)[e / 4], e);
                    } else {
                        for (int s = 0; s < splits; s += 4) {   // four ranges' loads at a time
                            float4 f[4][EU / 4];
#pragma unroll
                            for (int j = 0; j < 4; ++j)
#pragma unroll
                                for (int e = 0; e < EU / 4; ++e)
                                    f[j][e] = reinterpret_cast<const float4 *>(from + min(s + j, splits - 1) * step)[e];
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                if (s + j < splits)
#pragma unroll
                                    for (int e = 0; e < EU; e += 4) add(f[j][e / 4], e);
                        }
                    }
                }
                Unit<T> hi, lo;
#pragma unroll
                for (int e = 0; e < EU; ++e) {
                    if constexpr (PLANES == 1) {
                        hi.e[e] = v[e];
                    } else {
                        // what would round to an infinity: the largest bf16 value and the rest; of an infinity or NaN there is no rest
                        const bool finite = fabsf(v[e]) < INFINITY;
                        narrow(hi.e[e], finite ? fminf(fmaxf(v[e], -kLargest), kLargest) : v[e]);
                        narrow(lo.e[e], finite ? v[e] - widen(hi.e[e]) : 0.0f);
                    }
                }
                low[i][c][0] = hi.q;
                if constexpr (PLANES == 2) low[i][c][PLANES - 1] = lo.q;
            }
        }
    }
};

template <int MT> __device__ __forceinline__ void clear(f32x4 (&acc)[4][MT]) {
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int t = 0; t < MT; ++t) acc[q][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
}

// A wave's rows of y and the output: this lane has EU outputs, from col on, of the rows row + p RPL.
template <typename T, int MT> struct TileRows {
    static constexpr int EU = 16 / sizeof(T), TILE = 16 * MT, LPR = 64 / EU, RPL = 64 / LPR, PASSES = TILE / RPL;
    static constexpr int PITCH = 68;   // floats: 16 rows begin at different banks
    static constexpr int ROOM = TILE * PITCH;
    struct Rows {
        Unit<T> y[PASSES];
    };
    int row, col, end;
    bool on[PASSES];
    const T *yt[PASSES];
    T *ot[PASSES];
    __device__ __forceinline__ TileRows(const LowRankArgs &a, const TileTokens &tokens, int m1) {
        const int lane = threadIdx.x & 63;
        row = lane / LPR;
        col = lane % LPR * EU;
        end = m1;
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            on[p] = tokens.has(p * RPL + row);
            const long long t = tokens.token(p * RPL + row);
            yt[p] = static_cast<const T *>(a.y) + t * a.ys;
            ot[p] = static_cast<T *>(a.out) + t * a.os;
        }
    }
    __device__ __forceinline__ void load(Rows &s, int m) const {   // of outputs m on, or the last ones
#pragma unroll
        for (int p = 0; p < PASSES; ++p) s.y[p].q = *reinterpret_cast<const uint4 *>(yt[p] + min(m + col, end - EU));
    }
    // y and the products of outputs m on, acc[q][t] of block q and tokens 16 t.., by way of `room` in LDS, into the output
    // (ALL: all of these rows and outputs are there; a store under a condition would make the next wait for loads one for it too)
    template <bool ALL> __device__ __forceinline__ void store(const Rows &s, const f32x4 (&acc)[4][MT], int m, float *room) const {
        const int n16 = threadIdx.x & 15, h = (threadIdx.x & 63) >> 4;
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int q = 0; q < 4; ++q) *reinterpret_cast<f32x4 *>(room + (16 * t + n16) * PITCH + 16 * h + 4 * q) = acc[q][t];
        // (a wave's own LDS operations are in order)
        asm volatile("" ::: "memory");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            const float *at = room + (p * RPL + row) * PITCH + col;
            float add[EU];
#pragma unroll
            for (int e = 0; e < EU; e += 4) *reinterpret_cast<f32x4 *>(add + e) = *reinterpret_cast<const f32x4 *>(at + e);
            Unit<T> v;
#pragma unroll
            for (int e = 0; e < EU; ++e) narrow(v.e[e], widen(s.y[p].e[e]) + add[e]);
            if (ALL || (on[p] && m + col < end)) *reinterpret_cast<uint4 *>(ot[p] + m + col) = v.q;
        }
        asm volatile("" ::: "memory");
        __builtin_amdgcn_wave_barrier();
    }
};

// Tokens without an adapter: as they are.  By a whole wave.
template <typename T>
__device__ __forceinline__ void copy_rows(const LowRankArgs &a, const TileTokens &tokens, int tile, int m0, int m1) {
    constexpr int EU = 16 / sizeof(T);
    if (a.out == a.y) return;
    for (int i = 0; i < tile; ++i) {
        if (!tokens.has(i)) continue;
        const long long t = tokens.token(i);
        const T *y = static_cast<const T *>(a.y) + t * a.ys;
        T *out = static_cast<T *>(a.out) + t * a.os;
        for (int c = m0 + EU * (threadIdx.x & 63); c < m1; c += EU * 64)
            *reinterpret_cast<uint4 *>(out + c) = *reinterpret_cast<const uint4 *>(y + c);
    }
}

// Outputs m0 on up to m1, in `steps` of 64, of a tile's tokens with an adapter, by a wave.  load_low: h, after the first loads (EARLY)
// or before them.
template <typename T, int MT, int RC, bool GROUPED, bool EARLY, typename F>
__device__ __forceinline__ void expand_tile(const LowRankArgs &a, int adapter, const TileTokens &tokens, int m0, int m1, int steps, float *room,
                                            F load_low) {
    using C = Chunk<T>;
    using Tile = TileRows<T, MT>;
    using Rows = typename Tile::Rows;
    constexpr int EU = C::EU, TILE = 16 * MT;
    const int lane = threadIdx.x & 63, n16 = lane & 15, h = lane >> 4;
    const int rank = used_rank(a, adapter);
    const T *bt = static_cast<const T *>(a.b) + adapter * a.bs[0];
    const Tile rows(a, tokens, m1);
    uint4 b[RC][4];
    // Block q of B of step i, read again for the next step as soon as it is multiplied: half of the registers that two steps' B would
    // take (64 fp32 tokens of 38 adapters of rank 88: 30 to 25 us; 900 tokens of rank 104 in bf16, which have two waves to a
    // SIMD then: 13.7 to 9.2).  Of steps past the last, of that one again, so that no load is under a condition.
    auto load_b = [&](int q, int i) __attribute__((always_inline)) {
        const int m = m0 + 64 * min(i, max(steps - 1, 0));
#pragma unroll
        for (int c = 0; c < RC; ++c)   // rows past the last: that one, for nobody; past the rank: cleared below, as h is
            b[c][q] = *reinterpret_cast<const uint4 *>(bt + min(m + output_row(n16, q), m1 - 1) * a.bs[1] +
                                                       min((4 * c + h) * EU, a.rank - EU));
    };
    Low<T, MT, RC> low;
    Rows y0, y1;
    if constexpr (!EARLY) load_low(low);
    rows.load(y0, m0);
#pragma unroll
    for (int q = 0; q < 4; ++q) load_b(q, 0);
    if constexpr (EARLY) load_low(low);
    const int edge = rank / C::VALUES;   // the chunk that the rank ends in, and what of it counts
    const uint4 inside = within_rank<T>(make_uint4(~0u, ~0u, ~0u, ~0u), (4 * edge + h) * EU, rank);
    auto go = [&](auto all) __attribute__((always_inline)) {
        auto step = [&](int i, const Rows &now, Rows &later) __attribute__((always_inline)) {
            rows.load(later, m0 + 64 * min(i + 1, max(steps - 1, 0)));
            f32x4 acc[4][MT];
            clear(acc);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
#pragma unroll
                for (int c = 0; c < RC; ++c) {
                    if (c >= edge) {
                        b[c][q].x &= c == edge ? inside.x : 0;
                        b[c][q].y &= c == edge ? inside.y : 0;
                        b[c][q].z &= c == edge ? inside.z : 0;
                        b[c][q].w &= c == edge ? inside.w : 0;
                    }
                    low.multiply(acc, c, q, b[c][q]);
                }
                load_b(q, i + 1);
                __builtin_amdgcn_sched_barrier(0);
            }
            rows.template store<decltype(all)::value>(now, acc, m0 + 64 * i, room);
        };
#pragma unroll 1
        for (int i = 0; i < steps; ++i) {
            step(i, y0, y1);
            y0 = y1;
        }
    };
    if (GROUPED && tokens.count == TILE && (m1 - m0) % 64 == 0) go(std::true_type{});
    else go(std::false_type{});
}

// Every wave for itself: grouped, a workgroup's have four tiles of a span of outputs, whose B they find in the first-level cache
// (in LDS, with a barrier for every 64 outputs, it took 34 us where this takes 30: 8192 tokens, 4096 outputs, rank 16, bf16; rank 64 the same);
// else four spans of a tile.
template <typename T, int MT, int RC, bool GROUPED>
__global__ __launch_bounds__(256, MT * RC * (int)sizeof(T) <= 8 ? 2 : 1) void expand_kernel(LowRankArgs a) {
    constexpr int TILE = 16 * MT;
    __shared__ __align__(16) float room[4][TileRows<T, MT>::ROOM];
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned x1 = div_by(blockIdx.x, a.div_spans), x2 = div_by(x1, a.div_expand_ways);
    const long long at = blockIdx.x - x1 * a.div_spans.d, span = GROUPED ? at : 4 * at + w;
    const int m0 = (int)min(span * a.columns, (long long)a.m), m1 = (int)min((span + 1) * a.columns, (long long)a.m);
    if (m0 >= m1) return;
    auto tile_of = [&](int adapter, const TileTokens &tokens) __attribute__((always_inline)) {
        if (adapter < 0) return copy_rows<T>(a, tokens, TILE, m0, m1);
        expand_tile<T, MT, RC, GROUPED, true>(a, adapter, tokens, m0, m1, (m1 - m0 + 63) / 64, room[w], [&](auto &low) __attribute__((always_inline)) {
            low.load(a, a.splits, [&](int i) { return a.low + (long long)tokens.token(i) * a.rank; });
        });
    };
    if constexpr (GROUPED) {
        const int tile = 4 * (int)x2 + w, part = (int)div_by(tile, a.div_slots);
        if (tile - part * a.slots >= a.counts[part]) return;
        const int4 r = a.records[tile];
        tile_of(uniform(r.x), TileTokens{uniform(r.y), uniform(r.z), 0, a.grouped});
    } else {
        each_adapter<TILE>(a, (int)x2, (int)(x1 - x2 * a.expand_ways), a.expand_ways, tile_of);
    }
}

// Both at once, for calls so small that a launch counts: every workgroup has h of its tile's tokens for itself, in LDS, and
// its waves have spans of outputs, the first of which are on their way meanwhile.  One token of 4096 channels and 6144 outputs,
// rank 16, bf16: 9.0 us, the two launches 3.8 and 4.4; but a call from the host, which two launches and a workspace take
// 13 us, takes 8.6.
template <typename T, int NB> __global__ __launch_bounds__(64 * kShrinkWaves) void both_kernel(LowRankArgs a) {
    using S = Shrink<T, 1, NB>;
    constexpr int RC = (16 * NB + Chunk<T>::VALUES - 1) / Chunk<T>::VALUES, PITCH = S::RANK + 4;
    extern __shared__ __align__(16) float sums[];   // and then the waves' rooms; then h
    float *const low_at = sums + std::max(S::SUMS, S::W * TileRows<T, 1>::ROOM);
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned x1 = div_by(blockIdx.x, a.div_spans), x2 = div_by(x1, a.div_expand_ways);
    const long long span = (long long)S::W * (blockIdx.x - x1 * a.div_spans.d) + w;
    const int from = (int)min(span * a.columns, (long long)a.m), m1 = (int)min((span + 1) * a.columns, (long long)a.m);
    const int steps = (m1 - from + 63) / 64, m0 = steps ? from : 0;   // (a wave without outputs takes part in h)
    each_adapter<16>(a, (int)x2, (int)(x1 - x2 * a.expand_ways), a.expand_ways, [&](int adapter, const TileTokens &tokens) __attribute__((always_inline)) {
        if (adapter < 0) return copy_rows<T>(a, tokens, 16, from, m1);
        // (the first outputs' loads beside the products with A, where registers hold both)
        expand_tile<T, 1, RC, false, NB * (int)sizeof(T) <= 8>(a, adapter, tokens, m0, m1, steps, sums + w * TileRows<T, 1>::ROOM, [&](auto &low) __attribute__((always_inline)) {
            S::parts(a, adapter, tokens, 0, 0, sums);
            const int rank = used_rank(a, adapter);
            const float s = a.scales ? a.scales[adapter] : 1.0f;
            for (int i = threadIdx.x; i < 16 * S::RANK; i += 64 * S::W) {
                const int r = i % S::RANK;
                low_at[i / S::RANK * PITCH + r] = r < rank ? s * S::sum(sums, i) : 0.0f;
            }
            __syncthreads();
            low.load(a, 1, [&](int i) { return low_at + i * PITCH; });
        });
    });
}

template <typename T, int MT, int NB, bool GROUPED> hipError_t shrink_go(const LowRankPlan &pl, const LowRankArgs &a, hipStream_t st) {
    constexpr int LDS = GROUPED ? Ring<T, MT, NB>::LDS : kShrinkWaves * 16 * MT * 16 * NB * (int)sizeof(float);
    void (*kernel)(LowRankArgs);
    if constexpr (GROUPED) kernel = shrink_ring_kernel<T, MT, NB>;
    else kernel = shrink_kernel<T, MT, NB>;
    if constexpr (LDS > 65536) {
        static std::atomic<uint64_t> raised{0};   // devices whose limit is raised for this kernel
        const hipError_t err = raise_lds_limit(reinterpret_cast<const void *>(kernel), LDS, raised);
        if (err != hipSuccess) return err;
    }
    kernel<<<(unsigned)pl.tiles * pl.ways * pl.splits * pl.groups, GROUPED ? 256 : 64 * kShrinkWaves, LDS, st>>>(a);
    return hipGetLastError();
}
template <typename T, int MT, bool GROUPED> hipError_t go(const LowRankPlan &pl, const LowRankArgs &a, hipStream_t st) {
    const hipError_t err = pl.blocks == 1   ? shrink_go<T, MT, 1, GROUPED>(pl, a, st)
                           : pl.blocks == 2 ? shrink_go<T, MT, 2, GROUPED>(pl, a, st)
                           : pl.blocks == 4 ? shrink_go<T, MT, 4, GROUPED>(pl, a, st)
                                            : shrink_go<T, MT, 8, GROUPED>(pl, a, st);
    if (err != hipSuccess) return err;
    const unsigned blocks = (unsigned)((pl.tiles + pl.together - 1) / pl.together) * pl.expand_ways * pl.spans;
    auto expand = [&](auto chunks) {
        constexpr int RC = decltype(chunks)::value;
        expand_kernel<T, MT, RC, GROUPED><<<blocks, 256, 0, st>>>(a);
        return hipGetLastError();
    };
    constexpr int V = Chunk<T>::VALUES;
    if (a.rank <= V) return expand(std::integral_constant<int, 1>{});
    if (a.rank <= 2 * V) return expand(std::integral_constant<int, 2>{});
    if (sizeof(T) == 2 || a.rank <= 4 * V) return expand(std::integral_constant<int, 4>{});
    if constexpr (sizeof(T) == 4) return expand(std::integral_constant<int, 8>{});
    return hipErrorInvalidValue;   // (no rank is so large)
}
template <typename T, int NB> hipError_t both_go(const LowRankPlan &pl, const LowRankArgs &a, hipStream_t st) {
    using S = Shrink<T, 1, NB>;
    constexpr int LDS = (std::max(S::SUMS, S::W * TileRows<T, 1>::ROOM) + 16 * (S::RANK + 4)) * (int)sizeof(float);
    if constexpr (LDS > 65536) {
        static std::atomic<uint64_t> raised{0};   // devices whose limit is raised for this kernel
        const hipError_t err = raise_lds_limit(reinterpret_cast<const void *>(both_kernel<T, NB>), LDS, raised);
        if (err != hipSuccess) return err;
    }
    both_kernel<T, NB><<<(unsigned)pl.tiles * pl.expand_ways * pl.spans, 64 * S::W, LDS, st>>>(a);
    return hipGetLastError();
}
template <typename T> hipError_t pick(const LowRankPlan &pl, const LowRankArgs &a, hipStream_t st) {
    if (pl.both) {
        if constexpr (sizeof(T) == 2)
            if (pl.blocks == 8) return both_go<T, 8>(pl, a, st);
        if (pl.blocks == 4) return both_go<T, 4>(pl, a, st);
        return pl.blocks == 1 ? both_go<T, 1>(pl, a, st) : both_go<T, 2>(pl, a, st);
    }
    if (pl.grouped) return pl.tile == 16 ? go<T, 1, true>(pl, a, st) : go<T, 2, true>(pl, a, st);
    return pl.tile == 16 ? go<T, 1, false>(pl, a, st) : go<T, 2, false>(pl, a, st);
}

// Calls of one launch: so many tokens, bytes that a workgroup reads for a tile's h, and all of them do, and bytes of a row of B,
// past which registers spill.
constexpr int kBothTokens = 512, kBothRank = 256;
constexpr long long kBothBytes = 1 << 18, kBothAll = 24 << 20;

// Bins of group_kernel, two counts each, that LDS holds without more of it being asked for.
constexpr int kMaxBins = 8000;

}  // namespace

LowRankPlan low_rank_plan(const ftcnn_low_rank_desc &d) {
    LowRankPlan p{};
    if (d.tokens == 0) return p;
    // Grouping the tokens is a launch (3.5 us) more.  It pays where tiles of 16 neighbours read much of the weights, each of them
    // what all adapters have at most, or 16 of them: 48 MB.  128 tokens of 4096 channels and outputs in bf16, apart and grouped:
    // 4 adapters of rank 16 (8 MB) 9.7 and 12.8 us, 32 of them (29 MB) 14 and 14, 8 of rank 64 (67 MB) 19.5 and 17; 300 tokens of
    // those 8 (159 MB) 36 and 20.
    const double read = (d.tokens + 15) / 16 * (double)std::min(16, d.adapters) * d.rank * ((double)d.ch + d.m) * (d.dtype == FTCNN_F32 ? 4 : 2);
    p.grouped = read > 48 << 20 && d.adapters < kMaxBins;
    // two tiles of 16 together where they fill the device and adapters have as many tokens
    p.tile = d.tokens >= 32 * kComputeUnits / 2 && d.tokens / d.adapters >= 32 ? 32 : 16;
    p.tiles = (d.tokens + p.tile - 1) / p.tile;
    if (p.grouped) {
        // a part's tiles: every bin (an adapter, or none) has one that is not full at most, and all of them are full up to one
        p.parts = (d.tokens + kPart - 1) / kPart;
        p.slots = (std::min(kPart, d.tokens) + p.tile - 1) / p.tile + std::min(d.adapters, kPart);
        p.slots = (p.slots + 3) / 4 * 4;   // the second launch's workgroups have four tiles of a part
        p.tiles = p.parts * p.slots;
    }
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
    p.splits = (int)std::max(1LL, std::min(chunks / (4 * kShrinkWaves), (p.grouped ? 1LL : 2LL) * kComputeUnits / ((long long)p.tiles * p.groups * p.ways)));
    // One launch where every workgroup can have its tile's h for itself: 256 KB to read for it at most, and 24 MB for all tiles,
    // adapters and spans of outputs.  (From the host; with two launches each takes 12 to 13 us: 16 tokens of 4096 channels and
    // rank 16, 256 KB, 10.6; 512 tokens of 128 channels and outputs, 8 adapters of rank 16, 8.2; of 1024 and 2048, rank 32,
    // 100 MB, 15.9, and 13.5 with two.)
    const long long es = d.dtype == FTCNN_F32 ? 4 : 2, low = (d.rank + std::min(d.tokens, 16)) * (long long)d.ch * es;
    if (!p.grouped && d.tokens <= kBothTokens && d.rank * es <= kBothRank && low <= kBothBytes) {
        const long long waves = ((d.m + 63) / 64 + kShrinkWaves - 1) / kShrinkWaves;
        const int ways = share(kComputeUnits, p.tiles);
        const long long most_spans = std::max(1LL, std::min(waves, 2LL * kComputeUnits / ((long long)p.tiles * ways)));
        const long long each = (waves + most_spans - 1) / most_spans, spans = (waves + each - 1) / each;
        p.both = p.tiles * std::min<long long>(most, d.tokens) * spans * low <= kBothAll;
        if (p.both) {
            p.blocks = rows > 4 ? 8 : (rows > 2 ? 4 : rows);
            p.groups = p.splits = p.together = 1;
            p.expand_ways = ways;
            p.columns = (int)(64 * each);
            p.spans = (int)spans;
            return p;
        }
    }
    // The second launch: as many spans of 64 outputs as fill two workgroups to a compute unit, and no second round of them.
    const long long blocks = (d.m + 63) / 64;
    p.together = p.grouped ? 4 : 1;
    p.expand_ways = share(2 * kComputeUnits, p.tiles);
    const long long rows_of = (p.tiles + p.together - 1) / p.together * (long long)p.expand_ways, wide = 4 / p.together;
    const long long spans = std::max(1LL, std::min((blocks + wide - 1) / wide, 2 * kComputeUnits / rows_of));
    const long long each = (blocks + spans * wide - 1) / (spans * wide);
    p.columns = (int)(64 * each);
    p.spans = (int)((blocks + each * wide - 1) / (each * wide));
    auto up = [](size_t x) { return (x + 255) & ~size_t(255); };
    p.records = up((size_t)p.splits * d.tokens * d.rank * sizeof(float));
    p.bytes = p.records;
    if (p.grouped) {
        p.order = p.records + up((size_t)p.tiles * sizeof(int4));
        p.count = p.order + up((size_t)d.tokens * sizeof(int32_t));
        p.bytes = p.count + up(p.parts * sizeof(int32_t));
    }
    return p;
}

hipError_t launch_low_rank(int dtype, const LowRankPlan &pl, const LowRankArgs &a, hipStream_t st) {
    if (pl.grouped) {
        group_kernel<<<pl.parts, kGroup, 2 * (a.adapters + 1) * sizeof(int), st>>>(a, pl.tile);
        const hipError_t err = hipGetLastError();
        if (err != hipSuccess) return err;
    }
    return dtype == FTCNN_F32 ? pick<float>(pl, a, st) : pick<uint16_t>(pl, a, st);
}

}  // namespace ftcnn
