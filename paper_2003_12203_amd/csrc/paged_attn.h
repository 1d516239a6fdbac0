// Attention of new tokens over a paged cache of keys and values: the kernel.
//
//   S_ij = scale * q_i . k_j over the keys j that row i sees,
//   O_i = sum_j exp(S_ij - m_i) v_j / l_i,  l_i = sum_j exp(S_ij - m_i),  m_i = max_j S_ij,
//
// in one pass over the keys with the running maximum m and sum l, all of these in fp32 (powers of
// two: exp(x) = 2^(x log2 e)).  Rows are (new token, query head of one key head) pairs, so all the
// queries that share a key head share its loads; a workgroup of WR waves owns 32 WR rows and walks the
// keys in tiles of 32 KS, which 16-byte loads move straight into LDS, one tile ahead.
//
// The products run transposed.  S^T = K Q^T has a row's scores in one lane and its other half
// (lane ^ 32): softmax needs one exchange.  A lane then holds the keys 8 q + 4 half + (0..3), and
// O^T = V^T P^T takes any order of its keys as long as both operands have the same: P stays in
// registers, rounded to bf16 (fp32 kernels: as it is), and V is read from LDS in that order (bf16:
// transposed on the way, four keys of 16 columns at a time).  That rounding is what the bf16 matrix instructions ask
// for; the fp32 ones would hold every bit at an eighth of their rate.  The sum takes the unrounded weights.  Outputs
// of two prompts are within 0.0020 of float64, relative and root mean square, where exact weights leave 0.0015, the
// outputs' own rounding.
//
// LDS rows are unpadded (the direct loads write 1024 consecutive bytes a wave); 16-byte units are
// permuted within a row instead, so that what a cycle reads falls on different banks: the loads fetch
// the unit that belongs at their place.
//
// Schedules.  A unit is a tile of rows of one key head of one sequence.  "Whole": a workgroup a unit.
// "Even": the units, one after the other, each as long as the keys its rows see and what its start
// costs, are cut into equal runs, one a workgroup, so that the device is busy to the end whatever the
// lengths, which only the device knows; a unit that spans several runs is joined by a second launch
// (attn_join_kernel).
//
// What bounds it, with many rows, is the matrix cores and what keeps them from being fed: the weights (an
// exponential and its rounding for 4 dim operations) and the waits.  The scores of the next tile are multiplied
// while this one's weights are made (one prompt's tile after the other 1157 us, so 1102), in an order written
// by hand with scalar page addresses (1034).  Two prompts of 8192 tokens, 32 heads of 128 over eight key heads,
// causal, bf16: 1050 to 1085 us on several devices, 1010 to 1050 TFLOP/s of the 1260 that a product of 8192 x 8192
// matrices reaches; a rise of the matrix cores' share from 45 to 55 % took the clock from 2.13 to 1.87 GHz, so the
// power limit is near as well.  Chunks over 8192 cached tokens take twice their floor: the cut units' parts are
// written, read and joined (64 MB), and a workgroup's start is five tiles long.  fp32, a prompt of 4096 tokens, 32
// heads over eight key heads: 116 TFLOP/s of 153 with heads of 64, 122 with 128, 112 with 256.  Whole units are
// dealt out once, without a look at who is done: where they are about two to a compute unit, the longest may meet on
// one (16 heads over 16 or four: 66 TFLOP/s).
#pragma once

#include <limits.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "paged.h"

namespace ftcnn {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// Sixteen bytes a lane from memory (base + the lane's offset) straight into LDS at `to` + 16 lane; lanes that are
// switched off leave theirs as it is.  The compiler makes every later read of LDS wait for such loads if it
// knows of them, reads of the tile being worked on as well: it does not here, so the kernels wait (wait_loads)
// before the barrier that hands a tile over.
__device__ __forceinline__ void load_to_lds(const char *base, unsigned offset, unsigned to) {
    unsigned m0;   // the compiler's, put back
    const unsigned long long at = reinterpret_cast<unsigned long long>(base);
    const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)at), hi = __builtin_amdgcn_readfirstlane((unsigned)(at >> 32));
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2\n\ts_mov_b32 m0, %0"
                 : "=&s"(m0)
                 : "v"(offset), "s"((unsigned long long)hi << 32 | lo), "s"(__builtin_amdgcn_readfirstlane(to))
                 : "memory");
}
__device__ __forceinline__ void load_to_lds(const char *from, unsigned to) {
    unsigned m0;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off\n\ts_mov_b32 m0, %0"
                 : "=&s"(m0)
                 : "v"(from), "s"(__builtin_amdgcn_readfirstlane(to))
                 : "memory");
}
// All of this wave's loads have landed; then all of the workgroup's.
__device__ __forceinline__ void wait_loads() {
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
    asm volatile("" ::: "memory");
}
__device__ __forceinline__ void tile_barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// A value that all lanes agree on, in scalar registers.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ long long uniform(long long x) {
    return (long long)((unsigned long long)(unsigned)uniform((int)(x >> 32)) << 32 | (unsigned)uniform((int)x));
}

// A sequence: its new tokens [q0, q0 + nq) and cached tokens, within what the caller's arrays hold, and
// its units: row_tiles tiles of `rows` rows for each key head.  What row tile t costs is in keys: those it
// may see at most, cost0 + (t + 1) slope, with a.unit_cost for its start.
struct AttnSeq {
    int q0, nq, kv;
    int row_tiles, cost0, slope;
    __device__ AttnSeq(const AttnArgs &a, int b, int rows) {
        if (a.q_starts) {
            q0 = min(max(a.q_starts[b], 0), a.tokens);
            nq = min(max(a.q_starts[b + 1], q0), a.tokens) - q0;
        } else {
            q0 = b;
            nq = 1;
        }
        kv = min(max(a.kv_lens[b], 0), a.capacity);
        row_tiles = (nq * a.group + rows - 1) / rows;
        const int of_tile = min(nq, (rows + a.group - 2) / a.group + 1);   // tokens of a tile, at most
        int most = kv;
        slope = 0;
        if (a.window > 0) {   // from the first token's first key to the last one's own
            most = min(kv, a.window + of_tile - 1);
        } else if (a.causal && row_tiles > 1) {
            most = max(0, kv - nq);
            slope = of_tile;
        }
        cost0 = a.unit_cost + (most + a.tile_keys - 1) / a.tile_keys * a.tile_keys;
    }
    // (of a sequence that all lanes agree on)
    __device__ __forceinline__ void settle() {
        q0 = uniform(q0);
        nq = uniform(nq);
        kv = uniform(kv);
        row_tiles = uniform(row_tiles);
        cost0 = uniform(cost0);
        slope = uniform(slope);
    }
    // the keys [lo, hi) that the rows of tokens i0..i1 see, from a multiple of 16 on
    __device__ void range(const AttnArgs &a, int i0, int i1, int &lo, int &hi) const {
        const int past = kv - nq;
        hi = a.causal ? min(kv, max(0, past + i1 + 1)) : kv;
        lo = a.window > 0 ? min(hi, max(0, past + i0 - a.window + 1)) & ~15 : 0;
    }
    __device__ int cost(int t) const { return cost0 + (t + 1) * slope; }
    // the costs of row tiles 0..t - 1, of a key head's units, and of all
    __device__ long long before(int t) const { return (long long)t * cost0 + (long long)slope * ((long long)t * (t + 1) / 2); }
    __device__ long long head_work() const { return before(row_tiles); }
    __device__ long long work(const AttnArgs &a) const { return a.kv_heads * head_work(); }
    // the row tile that cost y < head_work() of a key head falls in
    __device__ int find(long long y) const {
        int t = 0, end = row_tiles;
        while (end - t > 1) {
            const int mid = (t + end) / 2;
            if (before(mid) <= y) t = mid;
            else end = mid;
        }
        return t;
    }
};

// a / b of what is not negative, in 32 bits where they hold it (the wide division takes a microsecond).
__device__ __forceinline__ long long divide(long long a, long long b) {
    if (((a | b) >> 32) == 0) return (unsigned)a / (unsigned)b;
    return a / b;
}

// The even schedule: the run (of the units' costs) a workgroup takes, and where a sequence's units begin.
struct AttnRuns {
    long long total, run;
    long long upto;   // the work of the sequences up to this lane's, of the first 64: the whole of them mostly
    __device__ static long long scan(const AttnArgs &a, int rows, int b) {
        const int lane = threadIdx.x & 63;
        long long incl = b < a.batch ? AttnSeq(a, b, rows).work(a) : 0;
#pragma unroll
        for (int x = 1; x < 64; x *= 2) {
            const long long v = __shfl_up(incl, x);
            if (lane >= x) incl += v;
        }
        return incl;
    }
    // by a whole wave
    __device__ AttnRuns(const AttnArgs &a, int rows) {
        const int lane = threadIdx.x & 63;
        upto = scan(a, rows, lane);
        long long sum = __shfl(upto, 63);
        if (a.batch > 64) {
            long long more = 0;
            for (int b = 64 + lane; b < a.batch; b += 64) more += AttnSeq(a, b, rows).work(a);
#pragma unroll
            for (int x = 32; x > 0; x /= 2) more += __shfl_xor(more, x);
            sum += more;
        }
        total = uniform(sum);
        run = max(divide(total + a.groups - 1, a.groups), (long long)a.min_run);
    }
    // the sequence that cost `at` < total belongs to, and where that sequence begins
    __device__ int find(const AttnArgs &a, int rows, long long at, long long &base) const {
        const int lane = threadIdx.x & 63;
        base = 0;
        for (int b0 = 0;; b0 += 64) {
            const long long incl = b0 == 0 ? upto : scan(a, rows, b0 + lane);
            const unsigned long long past = __ballot(base + incl > at);
            if (past || b0 + 64 >= a.batch) {
                const int at_lane = past ? __builtin_ctzll(past) : 63;
                base += at_lane > 0 ? __shfl(incl, max(at_lane - 1, 0)) : 0;
                return min(b0 + at_lane, a.batch - 1);
            }
            base += __shfl(incl, 63);
        }
    }
};

// Values that a row must not take up: a key that it does not see has weight zero, but zero times an infinity or NaN is
// NaN.  Tiles that some row (of the workgroup, which shares them) does not see all of are searched for such values, which
// are set to zero in them; a unit that had any gets them back at its end, added to the rows that see them, once.  In the
// other tiles they are multiplied as they are; that one of these may get a value a second time changes nothing of
// a sum that is infinite or NaN.  Every wave searches such a tile before it reads it, so that no result hangs on which
// wave came first.
template <typename T> struct NonFinite;
template <> struct NonFinite<uint16_t> {   // two values a word: the carry of a full exponent reaches its sign
    __device__ static uint32_t find(uint32_t w) { return (w & 0x7f807f80u) + 0x00800080u; }
    __device__ static bool any(uint32_t found) { return found & 0x80008000u; }
    __device__ static uint32_t clear(uint32_t w) {
        const uint32_t f = find(w);
        return w & ~(((f >> 15) & 1u) * 0x0000ffffu | (f >> 31) * 0xffff0000u);
    }
};
template <> struct NonFinite<float> {
    __device__ static uint32_t find(uint32_t w) { return (w & 0x7f800000u) + 0x00800000u; }
    __device__ static bool any(uint32_t found) { return found & 0x80000000u; }
    __device__ static uint32_t clear(uint32_t w) { return any(find(w)) ? 0u : w; }
};
__device__ inline float value_of(uint16_t v) { return bf16_bits_to_f32(v); }
__device__ inline float value_of(float v) { return v; }

// Clears what is not finite of a word, and says whether there was any.
template <typename T> __device__ __forceinline__ bool wash(uint32_t &w) {
    const bool any = NonFinite<T>::any(NonFinite<T>::find(w));
    if (any) w = NonFinite<T>::clear(w);
    return any;
}

// The offset of a row of a page, in bytes.
__device__ __forceinline__ unsigned long long page_row(int page, unsigned page_bytes, int row, unsigned row_bytes) {
    return (unsigned long long)(unsigned)page * page_bytes + (unsigned long long)(unsigned)row * row_bytes;
}
// Where workgroup g puts a unit's part that it holds only partly: slot 0 if the unit began in an earlier
// run, slot 1 if it began in this one.
__device__ inline long long attn_part(long long g, bool began_here) { return 2 * g + (began_here ? 1 : 0); }

// Calls unit(sequence, its number, key head, row tile, from, to, part) for all that this workgroup has to do: the
// unit's keys from its first + `from` to its first + `to`, or to its last where that is less; part < 0: they are
// the whole unit.
template <bool EVEN, typename F>
__device__ __forceinline__ void attn_schedule(const AttnArgs &a, int rows, int keys, F unit) {
    if constexpr (!EVEN) {   // whole units; of a sequence's row tiles the last, with the most keys, first
        unsigned pair, in;
        if (a.interleave) {   // a (sequence, key head)'s workgroups on one XCD, whose L2 then holds its keys
            const unsigned s = blockIdx.x >> 3;
            pair = s / (unsigned)a.tiles * 8 + (blockIdx.x & 7);
            in = s % (unsigned)a.tiles;
        } else {
            pair = blockIdx.x / (unsigned)a.tiles;
            in = blockIdx.x % (unsigned)a.tiles;
        }
        const int b = (int)(pair / (unsigned)a.kv_heads), hk = (int)(pair % (unsigned)a.kv_heads);
        AttnSeq sq(a, b, rows);
        sq.settle();
        for (int rt = a.tiles - 1 - (int)in; rt < sq.row_tiles; rt += a.tiles) unit(sq, b, hk, rt, 0, INT_MAX, -1);
    } else {
        const AttnRuns runs(a, rows);
        // consecutive workgroups are on different XCDs: each XCD's take consecutive runs, whose row tiles
        // of one key head read the same keys
        const unsigned rest = gridDim.x % 8, x = blockIdx.x % 8, each = gridDim.x / 8;
        const unsigned g = x * each + min(x, rest) + blockIdx.x / 8;
        long long at = g * runs.run;
        const long long end = uniform(min(at + runs.run, runs.total));
        // what the join has to know: whether this run starts inside a unit, and which
        AttnCut *cut = a.cuts + g;
        if (at >= end) {
            if (threadIdx.x == 0) cut->first_run = -1;
            return;
        }
        long long base;
        int b = uniform(runs.find(a, rows, at, base));
        base = uniform(base);
        while (at < end) {
            AttnSeq sq(a, b, rows);
            sq.settle();
            const long long next = base + sq.work(a);
            if (at >= next) {   // the run goes on in a later sequence
                base = next;
                ++b;
                continue;
            }
            const long long of_head = sq.head_work();
            const int hk = uniform((int)divide(at - base, of_head));
            const long long y = at - base - hk * of_head;
            const int rt = uniform(sq.find(y)), cost = uniform(sq.cost(rt)), c0 = uniform((int)(y - sq.before(rt)));
            const int c1 = uniform((int)min((long long)cost, c0 + (end - at)));
            if (threadIdx.x == 0 && at == g * runs.run) {
                const long long first = at - c0;
                *cut = AttnCut{c0 == 0 ? -1 : (int)divide(first, runs.run), (int)divide(first + cost - 1, runs.run),
                               sq.q0, hk, rt * rows, min(rows, sq.nq * a.group - rt * rows)};
            }
            // whole key tiles, wherever the cut falls
            auto key = [&](int cst) { return (max(0, cst - a.unit_cost) + keys - 1) / keys * keys; };
            unit(sq, b, hk, rt, key(c0), c1 == cost ? INT_MAX : key(c1),
                 c0 == 0 && c1 == cost ? -1 : attn_part(g, c0 == 0));
            at = uniform(at + (c1 - c0));
        }
    }
}

__device__ __forceinline__ void store4(float *p, float4 v) { *reinterpret_cast<float4 *>(p) = v; }
__device__ __forceinline__ void store4(uint16_t *p, float4 v) {
    union { uint2 q; uint16_t e[4]; } b;
    b.e[0] = f32_to_bf16_rne(v.x);
    b.e[1] = f32_to_bf16_rne(v.y);
    b.e[2] = f32_to_bf16_rne(v.z);
    b.e[3] = f32_to_bf16_rne(v.w);
    *reinterpret_cast<uint2 *>(p) = b.q;
}

// Rows of no sequence, before q_starts[0] and from q_starts[batch] on (padding up to a captured step's size), are what
// rows that see nothing are: a caller's buffers hold anything.  The launch's workgroups share them.
template <typename T, int THREADS> __device__ __forceinline__ void attn_clear_unowned(const AttnArgs &a) {
    if (!a.q_starts) return;
    const int first = min(max(a.q_starts[0], 0), a.tokens), last = min(max(a.q_starts[a.batch], first), a.tokens);
    const int count = first + a.tokens - last, heads = a.kv_heads * a.group, col = 4 * (threadIdx.x % 64);   // dim <= 256
    for (int i = blockIdx.x; i < count; i += gridDim.x) {
        const long long token = i < first ? i : last + (i - first);
        T *row = static_cast<T *>(a.o) + token * a.os[0];
        if (col < a.dim)
            for (int head = threadIdx.x / 64; head < heads; head += THREADS / 64)
                store4(row + head * a.os[1] + col, make_float4(0.0f, 0.0f, 0.0f, 0.0f));
        if (a.lse)
            for (int h = threadIdx.x; h < heads; h += THREADS) a.lse[token * heads + h] = -INFINITY;
    }
}

template <typename T, int DP, int WR, int KS> struct AttnTile {
    static constexpr int THREADS = 64 * WR, ROWS = 32 * WR, KEYS = 32 * KS;
    static constexpr int EU = 16 / sizeof(T);          // values of a 16-byte unit
    static constexpr int UPR = DP / EU;                // units of a row
    static constexpr int RB = DP * (int)sizeof(T);     // bytes of a row
    static constexpr int SIDE = KEYS * RB;             // bytes of a tile of keys, or of values
    static constexpr int LOADS = KEYS * UPR / THREADS;
    static constexpr int LDS = 4 * SIDE + 16;          // keys and values, two tiles of each; `dirt`
    static_assert(KEYS * UPR % THREADS == 0 && LOADS > 0 && 64 % UPR == 0, "whole loads");
    // where unit u of row r lies: u ^ key_unit(r).  Keys: 16 lanes read the same unit of 16 consecutive rows.
    __device__ static int key_unit(int r) { return UPR == 8 ? (r >> 1) & 7 : r & 15; }
    // Values: 32 lanes read 64 bytes of four consecutive rows (bf16), or 128 bytes of rows r and r + 4.
    __device__ static int value_unit(int r) {
        if (sizeof(T) == 4) return ((r >> 2) & 1) << 3;
        return UPR == 8 ? ((r >> 1) & 1) << 2 : (r & 3) << 2;
    }
};

// One wave's 32 rows: a lane and lane ^ 32 hold a row.
template <typename T, int DP, int KS> struct AttnRows {
    static constexpr bool BF = sizeof(T) == 2;
    static constexpr int EU = 16 / sizeof(T), UPR = DP / EU, RB = DP * (int)sizeof(T), NQ = UPR / 2, ND = DP / 32;
    using L = AttnTile<T, DP, 1, KS>;
    uint4 qf[NQ];      // queries: unit 2 t + half of the row
    f32x16 o[ND];      // column n = lane % 32 of O^T: values d * 32 + 8 (e / 4) + 4 half + e % 4 of its row
    float m, l;        // maximum of the scores, unscaled; the sum over this lane's keys

    __device__ __forceinline__ void start(const T *row, int dim, int half) {
#pragma unroll
        for (int t = 0; t < NQ; ++t) {
            const int u = 2 * t + half;
            qf[t] = u * EU < dim ? *reinterpret_cast<const uint4 *>(row + u * EU) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[d][e] = 0.0f;
        m = -INFINITY;
        l = 0.0f;
    }

    typedef f32x16 Scores[KS];

    // S^T = K Q^T for the tile of keys at kt.
    __device__ __forceinline__ void scores(const unsigned char *kt, Scores &s) const {
        const int lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
            for (int e = 0; e < 16; ++e) s[ks][e] = 0.0f;
            const int row = ks * 32 + l32, f = L::key_unit(row);
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
    }

    // Scores of keys that a row does not see, of the tile of keys from j0 on; this row sees jlo..jhi.
    __device__ __forceinline__ void mask(Scores &s, int j0, int jlo, int jhi) const {
        const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int j = j0 + ks * 32 + 8 * (e / 4) + 4 * half + e % 4;
                s[ks][e] = j >= jlo && j <= jhi ? s[ks][e] : -INFINITY;
            }
    }
    // The largest score of this lane, and of the row's two lanes.
    __device__ __forceinline__ static float peak(const Scores &s) {
        float top = s[0][0];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, s[ks][e]);
        return top;
    }
    __device__ __forceinline__ static float both(float x) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    // The running maximum, moved only when a row's scores pass it by more than 2^8 (in the weights, which fp32 sums
    // hold as well): what was summed is then scaled.
    __device__ __forceinline__ void raise(float top, float c) {
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
    }

    // Scores become weights, and count in the sum.
    __device__ __forceinline__ void weights(Scores &s, float c) {
        const float mc = m == -INFINITY ? 0.0f : m * c;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                s[ks][e] = __builtin_amdgcn_exp2f(fmaf(s[ks][e], c, -mc));
                l += s[ks][e];
            }
    }

    // O^T += V^T P^T for the tile of values at vt.
    __device__ __forceinline__ void product(const unsigned char *vt, const Scores &s) {
        const int lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            if constexpr (BF) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    bf16x8_t p;
#pragma unroll
                    for (int e = 0; e < 8; ++e) p[e] = (__bf16)s[ks][8 * j + e];
                    // lane i of 16 reads four columns of key i / 4 and gets column i of four keys
                    const int i = lane & 15, key = ks * 32 + 16 * j + 4 * half + i / 4;
                    const int f = L::value_unit(4 * half + i / 4);   // the rest is a multiple of 8
#pragma unroll
                    for (int d = 0; d < ND; ++d) {
                        const int u = d * 4 + ((lane >> 4) & 1) * 2 + ((i & 3) >> 1);
                        const unsigned char *at = vt + key * RB + ((u ^ f) << 4) + (i & 1) * 8;
                        typedef __attribute__((address_space(3))) s16x4 lds4;
                        const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(at));
                        const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(at + 8 * RB));
                        const s16x8 v = {v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
                        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, v), p, o[d], 0, 0,
                                                                       0);
                    }
                }
            } else {
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int key = ks * 32 + 8 * (e / 4) + 4 * half + e % 4, f = half << 3;
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
    // Sets what is not finite in the tile of values to zero, and says whether there was any.
    __device__ __forceinline__ static bool wash_tile(unsigned char *vt) {
        uint32_t found = 0;
        uint4 *unit = reinterpret_cast<uint4 *>(vt) + (threadIdx.x & 63);
#pragma unroll 4
        for (int i = 0; i < KS * UPR / 2; ++i) {
            const uint4 w = unit[64 * i];
            found |= NonFinite<T>::find(w.x) | NonFinite<T>::find(w.y) | NonFinite<T>::find(w.z) | NonFinite<T>::find(w.w);
        }
        if (!__any(NonFinite<T>::any(found))) return false;
#pragma unroll 1
        for (int i = 0; i < KS * UPR / 2; ++i) {
            const uint4 w = unit[64 * i];
            unit[64 * i] = make_uint4(NonFinite<T>::clear(w.x), NonFinite<T>::clear(w.y), NonFinite<T>::clear(w.z),
                                      NonFinite<T>::clear(w.w));
        }
        return true;
    }
    // Adds what is not finite of the values of a key (at row), if this row sees it.
    __device__ __forceinline__ void restore(const T *row, int dim, bool seen) {
        const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                if (d * 32 + 2 * e < dim) {   // eight values of the head, of both halves
                    const T *at = row + d * 32 + 2 * e + 4 * half;
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const float v = value_of(at[x]);
                        o[d][e + x] += seen && !(fabsf(v) < INFINITY) ? v : 0.0f;
                    }
                }
    }

    // scores(kt, then), weights(now) and product(vt, now) in one, bf16, and peak(then): the matrix instructions in
    // a row, with LDS read AHEAD of them, and the vector unit's work between them, so that neither waits for the
    // other.  A product needs the weights of its 16 keys (group), so the first groups are made under the scores of
    // the next tile and the last under the products of the first.  A wave issues in order: an element's three
    // steps (argument, power, sum) are spread over three places.  beside(i): more to do after matrix instruction i.
    template <typename F>
    __device__ __forceinline__ float fused(const unsigned char *kt, const unsigned char *vt, Scores &now, Scores &then,
                                           float c, F beside) {
        constexpr int NS = NQ * KS, NG = 2 * KS, NP = NG * ND, AHEAD = 4;
        constexpr int WORK = 8 * NG + 2, BY = NS + (NG - 1) * ND;   // steps of the weights, and when they have to be done
        const int lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5, i16 = lane & 15;
        const unsigned char *krow = kt + l32 * RB;
        const int fk = L::key_unit(l32);   // rows 32 ks + l32: the same
        const unsigned char *vrow = vt + (4 * half + i16 / 4) * RB + (i16 & 1) * 8;
        const int fv = L::value_unit(4 * half + i16 / 4), uv = ((lane >> 4) & 1) * 2 + ((i16 & 3) >> 1);
        typedef __attribute__((address_space(3))) s16x4 lds4;
        s16x8 frag[AHEAD];
        auto read = [&](int i) __attribute__((always_inline)) {   // operand i: keys, then values
            if (i < NS) {
                const int ks = i % KS, x = i / KS;
                frag[i % AHEAD] = *reinterpret_cast<const s16x8 *>(krow + ks * 32 * RB + (((2 * x + half) ^ fk) << 4));
            } else if (i < NS + NP) {
                const int g = (i - NS) / ND, d = (i - NS) % ND;
                const unsigned char *at = vrow + 16 * g * RB + (((d * 4 + uv) ^ fv) << 4);
                const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(at));
                const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(at + 8 * RB));
                frag[i % AHEAD] = s16x8{v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
            }
        };
        const float mc = m == -INFINITY ? 0.0f : m * c;
        float top = -INFINITY;
        bf16x8_t pg[NG];
        auto work = [&](int k) __attribute__((always_inline)) {
            if (k >= 2) {
                const int e = k - 2;
                l += now[e / 16][e % 16];
                pg[e / 8][e % 8] = (__bf16)now[e / 16][e % 16];
            }
            if (k >= 1 && k <= 8 * NG) {
                const int e = k - 1;
                now[e / 16][e % 16] = __builtin_amdgcn_exp2f(now[e / 16][e % 16]);
            }
            if (k < 8 * NG) now[k / 16][k % 16] = fmaf(now[k / 16][k % 16], c, -mc);
        };
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int e = 0; e < 16; ++e) then[ks][e] = 0.0f;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) read(i);
#pragma unroll
        for (int i = 0; i < NS + NP; ++i) {
            const bf16x8_t f = __builtin_bit_cast(bf16x8_t, frag[i % AHEAD]);
            if (i < NS)
                then[i % KS] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, __builtin_bit_cast(bf16x8_t, qf[i / KS]),
                                                                       then[i % KS], 0, 0, 0);
            else
                o[(i - NS) % ND] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, pg[(i - NS) / ND], o[(i - NS) % ND], 0, 0, 0);
            read(i + AHEAD);
            const int done = i == 0 ? 0 : (i * WORK + BY - 1) / BY, to = ((i + 1) * WORK + BY - 1) / BY;
#pragma unroll
            for (int k = done; k < (to < WORK ? to : WORK); ++k) work(k);
            // the scores are complete a few instructions after the last of theirs
            if (i >= NS + 2) {
                constexpr int PER = (16 * KS + NP - 3) / (NP - 2);
#pragma unroll
                for (int k = (i - NS - 2) * PER; k < (i - NS - 1) * PER && k < 16 * KS; ++k)
                    top = fmaxf(top, then[k / 16][k % 16]);
            }
            beside(i);
            __builtin_amdgcn_sched_barrier(0);
        }
        return top;
    }

    // Four values of a row at a time, unit 8 e + 4 half of block d.
    template <typename F> __device__ __forceinline__ void each4(int dim, F f) const {
        const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int at = d * 32 + 8 * e + 4 * half;
                if (at < dim) f(at, make_float4(o[d][4 * e], o[d][4 * e + 1], o[d][4 * e + 2], o[d][4 * e + 3]));
            }
    }
};

// Two workgroups to a compute unit where registers hold them.  fp32, heads of 128, a prompt of 4096 tokens, 32 heads over eight
// key heads: 1118 us, one 1254; two of 8192 8.28 ms and 9.68; 1024 tokens, heads of 96: 112 and 118.  Not where the
// longest units meet: 16 heads over 16, 1037, one 694; over eight 766 and 649.
template <typename T, int DP, int WR, int KS, bool EVEN, bool ONE>
__global__ __launch_bounds__(64 * WR, DP > 128 ? 1 : 2) void attn_kernel(AttnArgs a) {
    using L = AttnTile<T, DP, WR, KS>;
    constexpr int UPR = L::UPR, EU = L::EU, RB = L::RB, OWN = L::KEYS / WR, STEP = 64 / UPR;   // rows of a wave's loads, of one
    extern __shared__ __align__(1024) unsigned char lds[];
    int *dirt = reinterpret_cast<int *>(lds + 4 * L::SIDE);   // the first and last tile of a unit with values not finite
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, half = lane >> 5;
    typedef __attribute__((address_space(3))) unsigned char lds_byte;
    const unsigned lds_at = (unsigned)(uintptr_t)(lds_byte *)lds;
    const float c = a.scale_log2;
    AttnRows<T, DP, KS> rows;
    if (DP != a.dim)   // the columns past the head, which no load writes
        for (int i = tid; i < 4 * L::SIDE / 16; i += L::THREADS) reinterpret_cast<uint4 *>(lds)[i] = make_uint4(0, 0, 0, 0);

    // As attn_schedule has it.
    auto unit = [&](const AttnSeq &sq, int b, int hk, int rt, int from, int to, long long part) __attribute__((always_inline)) {
        const int nrows = sq.nq * a.group, r0 = rt * L::ROWS;
        const int i0 = (int)div_by(r0, a.div_group), i1 = (int)div_by(min(r0 + L::ROWS, nrows) - 1, a.div_group);
        int lo, hi;
        sq.range(a, i0, i1, lo, hi);
        const int k0 = uniform(min(hi, lo + from)), k1 = uniform(to < hi - lo ? lo + to : hi);
        const int ntiles = k1 > k0 ? (k1 - k0 + L::KEYS - 1) / L::KEYS : 0;

        // this lane's row; past the last one, the last again (not stored)
        const int mine = r0 + w * 32 + l32, r = min(mine, nrows - 1);
        const bool idle = r0 + w * 32 >= nrows;
        const int qi = (int)div_by(r, a.div_group), head = hk * a.group + r - qi * a.group;
        const int pos = sq.kv - sq.nq + qi;
        const int jhi = min(a.causal ? pos : sq.kv - 1, k1 - 1);   // the keys it sees: jlo..jhi
        const int jlo = a.window > 0 ? pos - a.window + 1 : 0;
        // Of tiles [whole0, whole1) the workgroup's first row and its last one, so all of its rows, see every key.
        const int jhi_min = min(a.causal ? sq.kv - sq.nq + i0 : sq.kv - 1, k1 - 1);
        const int jlo_max = a.window > 0 ? sq.kv - sq.nq + i1 - a.window + 1 : 0;
        const int whole0 = uniform((max(jlo_max - k0, 0) + L::KEYS - 1) / L::KEYS);
        const int whole1 = uniform(max(jhi_min + 1 - k0, 0) / L::KEYS);
        rows.start(static_cast<const T *>(a.q) + (long long)(sq.q0 + qi) * a.qs[0] + (long long)head * a.qs[1], a.dim,
                   half);

        const char *kbase = static_cast<const char *>(a.k) + (long long)hk * a.kb[2];
        const char *vbase = static_cast<const char *>(a.v) + (long long)hk * a.vb[2];
        const int32_t *list = a.page_list + (long long)b * a.list_stride;
        // A wave loads rows w * OWN .. of a tile, load i this lane's unit of row own + i * STEP of these.  ONE: pages
        // hold a multiple of OWN rows, so that (tiles start at multiples of 16) a wave's are in one page, and their
        // addresses are scalars but for an offset of the lane.  Past a unit's last key, that one again.
        const int own = lane / UPR, slot = lane % UPR;
        constexpr int PIDS = ONE ? 1 : L::LOADS;
        int pid0[PIDS], pid1[PIDS];   // pages of an even and an odd tile
        auto key_of = [&](int t, int i) { return min(k0 + t * L::KEYS + w * OWN + own + i * STEP, k1 - 1); };
        auto lookup = [&](int t, int (&pid)[PIDS]) __attribute__((always_inline)) {
            if constexpr (ONE) {
                pid[0] = list[div_by_many(min(k0 + t * L::KEYS + w * OWN, k1 - 1), a.div_page)];
            } else {
#pragma unroll
                for (int i = 0; i < L::LOADS; ++i) pid[i] = list[div_by(key_of(t, i), a.div_page)];
            }
        };
        // One side of tile t into quarter t % 2 of LDS (keys), 2 + t % 2 (values).
        auto issue = [&](int t, const char *base, const unsigned (&bytes)[3], const int (&pid)[PIDS], bool values)
                         __attribute__((always_inline)) {
            const unsigned to = lds_at + ((values ? 2 : 0) + (t & 1)) * L::SIDE + w * OWN * RB;
            const int kw = min(k0 + t * L::KEYS + w * OWN, k1 - 1), last = k1 - 1 - kw;
            const char *page = base;
            if constexpr (ONE) {
                const int pg = min(max(__builtin_amdgcn_readfirstlane(pid[0]), 0), a.pages - 1);
                page += page_row(pg, bytes[0], kw - (int)div_by_many(kw, a.div_page) * a.page, bytes[1]);
            }
#pragma unroll
            for (int i = 0; i < L::LOADS; ++i) {
                const int row = own + i * STEP;
                const int u = slot ^ (values ? L::value_unit(w * OWN + row) : L::key_unit(w * OWN + row));
                if (DP != a.dim && u * EU >= a.dim) continue;   // past the head: LDS holds zeros there
                if constexpr (ONE) {
                    load_to_lds(page, __umul24(min(row, last), bytes[1]) + u * 16, to + i * 1024);
                } else {
                    const int key = key_of(t, i), in_page = key - (int)div_by(key, a.div_page) * a.page;
                    const int pg = min(max(pid[i], 0), a.pages - 1);
                    load_to_lds(page + page_row(pg, bytes[0], in_page, bytes[1]) + u * 16, to + i * 1024);
                }
            }
        };
        // The loop is one tile ahead with the scores: those of tile t + 1 go through the matrix cores while
        // the weights of tile t go through the vector unit.  So iteration t reads keys t + 1 and values t, and
        // has keys t + 2 and values t + 1 on their way into the halves of LDS that t - 1 has left.  Past the last
        // tile it multiplies what lies there, for nobody.
        // What is loaded past the last tile is not waited for in the loop, but before LDS is used again.
        wait_loads();
        __syncthreads();   // the unit before this one may still read LDS
        if (tid == 0) {
            dirt[0] = INT_MAX;
            dirt[1] = -1;
        }
        using Scores = typename AttnRows<T, DP, KS>::Scores;
        Scores s, next;   // of even and odd tiles
        float top = -INFINITY;
        if (ntiles > 0) {
            lookup(0, pid0);
            lookup(1, pid1);
            issue(0, kbase, a.kb, pid0, false);
            issue(0, vbase, a.vb, pid0, true);
            issue(1, kbase, a.kb, pid1, false);
            lookup(2, pid0);
            wait_loads();
            tile_barrier();
            rows.scores(lds, s);
            top = rows.peak(s);
        }
        auto tile = [&](int t, Scores &now, Scores &then, int (&mine)[PIDS], int (&other)[PIDS])
                        __attribute__((always_inline)) {
            wait_loads();
            tile_barrier();   // keys t + 1 and values t have landed, and nobody reads keys t or values t - 1 any more
            const unsigned char *kt = lds + ((t + 1) & 1) * L::SIDE, *vt = lds + (2 + (t & 1)) * L::SIDE;
            auto values = [&]() __attribute__((always_inline)) { issue(t + 1, vbase, a.vb, other, true); };
            auto keys = [&]() __attribute__((always_inline)) {
                issue(t + 2, kbase, a.kb, mine, false);
                lookup(t + 3, other);
            };
            if (idle) {
                values();
                keys();
                return;
            }
            if (t < whole0 || t >= whole1) {   // the whole workgroup: see NonFinite
                rows.mask(now, k0 + t * L::KEYS, jlo, jhi);
                top = rows.peak(now);
                if (rows.wash_tile(lds + (2 + (t & 1)) * L::SIDE) && lane == 0) {
                    atomicMin(&dirt[0], t);
                    atomicMax(&dirt[1], t);
                }
            }
            rows.raise(rows.both(top), c);
            if constexpr (sizeof(T) == 2 && ONE) {
                top = rows.fused(kt, vt, now, then, c, [&](int i) __attribute__((always_inline)) {
                    if (i == 0) values();
                    if (i == 4) keys();
                });
            } else if constexpr (sizeof(T) == 2) {
                values();
                keys();
                top = rows.fused(kt, vt, now, then, c, [](int) {});
            } else {
                values();
                keys();
                rows.scores(kt, then);
                rows.weights(now, c);
                rows.product(vt, now);
                top = rows.peak(then);
            }
        };
        for (int t = 0; t < ntiles; t += 2) {
            tile(t, s, next, pid0, pid1);
            if (t + 1 < ntiles) tile(t + 1, next, s, pid1, pid0);
        }
        __syncthreads();
        if (__builtin_expect(dirt[1] >= 0, 0)) {
            const int last = min(k1, k0 + (dirt[1] + 1) * L::KEYS);
#pragma unroll 1
            for (int key = k0 + dirt[0] * L::KEYS; key < last; ++key) {
                const int in = (int)div_by(key, a.div_page), pg = min(max(list[in], 0), a.pages - 1);
                const char *row = vbase + page_row(pg, a.vb[0], key - in * a.page, a.vb[1]);
                rows.restore(reinterpret_cast<const T *>(row), a.dim, key >= jlo && key <= jhi);
            }
        }
        const float m = rows.m, l = rows.l + __shfl_xor(rows.l, 32);
        const long long orow = (long long)(sq.q0 + qi) * a.kv_heads * a.group + head;
        if (mine >= nrows) return;
        if (part >= 0) {
            const long long at = part * a.part_rows + (mine - r0);
            float *po = a.part_o + at * a.dim;
            rows.each4(a.dim, [&](int x, float4 v) { *reinterpret_cast<float4 *>(po + x) = v; });
            if (half == 0) {
                a.part_ml[at * 2] = m * c;
                a.part_ml[at * 2 + 1] = l;
            }
            return;
        }
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;   // a row that sees nothing is zero
        T *out = static_cast<T *>(a.o) + (long long)(sq.q0 + qi) * a.os[0] + (long long)head * a.os[1];
        rows.each4(a.dim, [&](int x, float4 v) {
            store4(out + x, make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv));
        });
        if (a.lse && half == 0)
            a.lse[orow] = l == 0.0f ? -INFINITY : (m * c + __log2f(l)) * 0.693147180559945309f;
    };

    attn_schedule<EVEN>(a, L::ROWS, L::KEYS, unit);
    attn_clear_unowned<T, L::THREADS>(a);
}

// The limit is a device's own, so each device that the process launches on has it raised.
inline hipError_t raise_lds_limit(const void *kernel, int bytes, std::atomic<uint64_t> &raised) {
    int device = 0;
    hipError_t err = hipGetDevice(&device);
    if (err != hipSuccess) return err;
    const uint64_t bit = device < 64 ? 1ull << device : 0;
    if (raised.load(std::memory_order_relaxed) & bit) return hipSuccess;
    err = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (err == hipSuccess) raised.fetch_or(bit, std::memory_order_relaxed);
    return err;
}

template <typename T, int DP, int WR, int KS, bool EVEN, bool ONE>
hipError_t attn_launch(const AttnArgs &a, unsigned blocks, hipStream_t st) {
    using L = AttnTile<T, DP, WR, KS>;
    auto kernel = attn_kernel<T, DP, WR, KS, EVEN, ONE>;
    if constexpr (L::LDS > 65536) {
        static std::atomic<uint64_t> raised{0};   // devices whose limit is raised for this kernel
        const hipError_t err = raise_lds_limit(reinterpret_cast<const void *>(kernel), L::LDS, raised);
        if (err != hipSuccess) return err;
    }
    kernel<<<blocks, L::THREADS, L::LDS, st>>>(a);
    return hipGetLastError();
}
template <typename T, int DP, int WR, int KS> hipError_t attn_go(const AttnArgs &a, hipStream_t st) {
    // Page addresses in scalars (two prompts of 8192 tokens 1034 us, with an address a lane 1102), else one for every
    // load of a lane, which heads of 128 have no registers for (7 to 29 spilled): pages of 24 rows, bf16, two
    // prompts 1237 us (of 64: 1074), chunks over a cache 126 (115).
    const bool one = a.page % (AttnTile<T, DP, WR, KS>::KEYS / WR) == 0 && std::max(a.kb[1], a.vb[1]) < 1u << 24;
    const unsigned whole = (unsigned)a.tiles * a.kv_heads * a.batch;
    if (a.groups)
        return one ? attn_launch<T, DP, WR, KS, true, true>(a, a.groups, st)
                   : attn_launch<T, DP, WR, KS, true, false>(a, a.groups, st);
    return one ? attn_launch<T, DP, WR, KS, false, true>(a, whole, st)
               : attn_launch<T, DP, WR, KS, false, false>(a, whole, st);
}

}  // namespace ftcnn
