// The attention weight that every cached key gets from the new tokens:
//
//   mass_j += sum over rows i that see j of exp(scale q_i . k_j - L_i),
//
// with the rows' log-sums L given, so that the weights need no second pass over the keys.  Rows, sequences and masks
// are those of paged_attn.h.  The product is S^T = K Q^T: a lane has one row and several keys, whose weights it adds up
// over all rows and heads in registers; lanes are added at the end.  No order hangs on timing.
//
// mass_wide_kernel, more than 64 rows of a key head: a wave holds 64 keys of a head in registers (32 where heads are large, or
// where there would be too few workgroups), tiles of 64 rows (fewer where heads are large) go through LDS, which the
// workgroup's waves share, and the scores of the next 32 rows go through the matrix cores while these rows' weights are
// made.  What bounds it with many rows is the vector unit beside the matrix cores: for each weight an argument, a power and a
// sum, 16 cycles of it for every 16 that the matrix cores take for heads of 128, and the two overlap in part (by counters the matrix cores
// are busy for 51 % of the time, the vector unit, which issues for both, for 68 %).  Two prompts of 8192 tokens, 32 heads of 128 over eight key
// heads, bf16: 548 us, 1000 TFLOP/s of the 1260 that a product of 8192 x 8192 matrices reaches; as first written, with the weights after the
// scores, places divided for each row and lanes added through LDS, which spilled registers, 760.
// 49 tokens over 70440 keys, 64 heads of 96 over eight: 94 us (125 with a mask in every tile that is not full).
// Short calls pay for a workgroup's start, 8 us from its lengths to its sums.
//
// mass_few_kernel: the reading of the keys is all, straight into registers in the order of the matrix instructions; a
// wave takes every fourth head of a run of keys, the next head's keys on their way.  64 single tokens, ragged, over up
// to 8192 keys, 32 heads of 128 over eight, bf16, 102 MB: 25 us, 4.1 TB/s (a workgroup for every 64 keys that a sequence might have: 46; fp32,
// 204 MB: 50); one token over 131072, 268 MB: 54 us, 5.0 TB/s of the 5.2 of a large copy (fp32 108).  16 tokens of each of four sequences of 30016 keys (64 rows of a
// key head) 82 us, in the wide kernel 118.
#pragma once

#include "mass.h"
#include "paged_stream.h"

namespace ftcnn {

// A sequence: its new tokens [q0, q0 + nq) and cached tokens, within what the caller's arrays hold.
struct MassSeq {
    int q0, nq, kv;
    __device__ __forceinline__ MassSeq(const AttnArgs &a, int b) {
        q0 = b;
        nq = 1;
        if (a.q_starts) {
            q0 = min(max(a.q_starts[b], 0), a.tokens);
            nq = min(max(a.q_starts[b + 1], q0), a.tokens) - q0;
        }
        kv = min(max(a.kv_lens[b], 0), a.capacity);
    }
    // (of a sequence that all lanes agree on)
    __device__ __forceinline__ void settle() {
        q0 = uniform(q0);
        nq = uniform(nq);
        kv = uniform(kv);
    }
    // the first key that some row sees, to a multiple of 16, if one does
    __device__ __forceinline__ int first(const AttnArgs &a) const {
        return a.window > 0 ? min(kv, max(0, kv - nq - a.window + 1)) & ~15 : 0;
    }
};

// The new tokens [i0, i1) that may see a key of [k0, k1).
__device__ __forceinline__ void tokens_that_see(const AttnArgs &a, const MassSeq &sq, int k0, int k1, int &i0, int &i1) {
    const int past = sq.kv - sq.nq;
    i0 = a.causal ? min(max(k0 - past, 0), sq.nq) : 0;
    i1 = a.window > 0 ? min(max(k1 - 1 - past + a.window, 0), sq.nq) : sq.nq;
}

// This lane's row r (past the last one: sees nothing), what it sees, and where it is.
struct MassRow {
    int jlo, jhi, qi, head;
    __device__ __forceinline__ MassRow(const AttnArgs &a, const MassSeq &sq, int hk, int r) {
        const int nrows = sq.nq * a.group, at = min(r, nrows - 1);
        qi = (int)div_by(at, a.div_group);
        head = hk * a.group + at - qi * a.group;
        const int pos = sq.kv - sq.nq + qi;
        jhi = r < nrows ? (a.causal ? pos : sq.kv - 1) : -1;
        jlo = a.window > 0 ? pos - a.window + 1 : 0;
    }
};

// The sum over rows of 16 lanes, in all of them, by the vector unit alone.
template <int CTRL> __device__ __forceinline__ float with_lane(float x) {
    return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float sum16(float x) {
    x = with_lane<0xB1>(x);      // lane ^ 1
    x = with_lane<0x4E>(x);      // lane ^ 2
    x = with_lane<0x141>(x);     // the other four of eight
    return with_lane<0x140>(x);  // the other eight
}

// A wave's 32 KS keys of a head and what they got so far: lane and lane ^ 32 share a row, and have of each 32 keys those at
// 8 (e / 4) + 4 half + e % 4.
template <typename T, int DP, int KS> struct MassKeys {
    static constexpr bool BF = sizeof(T) == 2;
    static constexpr int EU = 16 / sizeof(T), UPR = DP / EU, NQ = UPR / 2;
    typedef f32x16 Scores[KS];
    uint4 kf[KS][NQ];       // unit 2 q + half of key 32 ks + lane % 32
    float got[KS][16];

    __device__ __forceinline__ static void multiply(f32x16 &s, uint4 k, uint4 q) {
        if constexpr (BF) {
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, k), __builtin_bit_cast(bf16x8_t, q), s, 0, 0, 0);
        } else {
            const float4 ka = __builtin_bit_cast(float4, k), qb = __builtin_bit_cast(float4, q);
            s = __builtin_amdgcn_mfma_f32_32x32x2f32(ka.x, qb.x, s, 0, 0, 0);
            s = __builtin_amdgcn_mfma_f32_32x32x2f32(ka.y, qb.y, s, 0, 0, 0);
            s = __builtin_amdgcn_mfma_f32_32x32x2f32(ka.z, qb.z, s, 0, 0, 0);
            s = __builtin_amdgcn_mfma_f32_32x32x2f32(ka.w, qb.w, s, 0, 0, 0);
        }
    }

    // Adds up the 32 lanes; lane l32 gets the sum of key l32 % (16 KS) of its own.
    __device__ __forceinline__ float sum() {
        const int mine = threadIdx.x & (16 * KS - 1);
        float res = 0.0f;
#pragma unroll
        for (int i = 0; i < 16 * KS; ++i) {
            float v = sum16(got[i / 16][i % 16]);
            v += __shfl_xor(v, 16);
            res = i == mine ? v : res;
        }
        return res;
    }

    // The scores `then` of the 32 rows at qt (this lane's row and its permutation f of units), and the weights of
    // the rows before them, `now`, added up: the matrix instructions in a row, LDS read AHEAD of them, and the vector unit's
    // work between them, an element's three steps (argument, power, sum) in three places.  MASKED: a key has a weight where
    // its place from the row's first key on (this lane's first one's: from) is at most span.
    template <bool MASKED>
    __device__ __forceinline__ void step(const unsigned char *qt, int f, Scores &now, Scores &then, float c, float log,
                                         unsigned from, unsigned span) {
        constexpr int NS = NQ * KS, AHEAD = 4, ELEMENTS = 16 * KS, WORK = ELEMENTS + 2;
        const int half = (threadIdx.x & 63) >> 5;
        uint4 frag[AHEAD];
        auto read = [&](int q) __attribute__((always_inline)) {
            if (q < NQ) frag[q % AHEAD] = *reinterpret_cast<const uint4 *>(qt + (((2 * q + half) ^ f) << 4));
        };
        auto work = [&](int k) __attribute__((always_inline)) {
            if (k >= 2) {
                const int e = k - 2;
                got[e / 16][e % 16] += now[e / 16][e % 16];
                // here, not behind the branch between masked and other rows, where 32 more registers would wait for it
                asm volatile("" : "+v"(got[e / 16][e % 16]));
            }
            if (k >= 1 && k <= ELEMENTS) {
                const int e = k - 1;
                now[e / 16][e % 16] = __builtin_amdgcn_exp2f(now[e / 16][e % 16]);
            }
            if (k < ELEMENTS) {
                float x = fmaf(now[k / 16][k % 16], c, -log);
                if constexpr (MASKED) {
                    x = from + (32 * (k / 16) + 8 * (k % 16 / 4) + k % 4) <= span ? x : -INFINITY;
                }
                now[k / 16][k % 16] = x;
            }
        };
#pragma unroll
        for (int q = 0; q < AHEAD; ++q) read(q);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int e = 0; e < 16; ++e) then[ks][e] = 0.0f;
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            multiply(then[i % KS], kf[i % KS][i / KS], frag[i / KS % AHEAD]);
            if (i % KS == KS - 1) read(i / KS + AHEAD);
            const int done = i * WORK / NS, to = (i + 1) * WORK / NS;
#pragma unroll
            for (int k = done; k < to; ++k) work(k);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
};

// How a tile's rows lie: those of one query head (by_head), or of all of the key head's, tokens' heads together, as 1 << shift of
// them divide a tile's rows (other groups, of few tokens: shift -1).  By heads (two prompts of 8192 tokens 581 us; tokens' heads
// together 595) unless the last tile of each, which is not full, would be another 15th.
template <int ROWS> struct MassOrder {
    bool by_head;
    int shift;
    __device__ __forceinline__ MassOrder(const AttnArgs &a, const MassSeq &sq) {
        shift = a.group <= ROWS && (a.group & (a.group - 1)) == 0 ? __builtin_ctz(a.group) : -1;
        const int apart = (sq.nq + ROWS - 1) / ROWS * a.group, together = (sq.nq * a.group + ROWS - 1) / ROWS;
        by_head = sq.nq >= ROWS && (shift < 0 || apart - together <= together / 15);
        if (by_head) shift = 0;
    }
};
// The rows of a sequence that may see keys of [k0, k1), in tiles of ROWS.
template <int ROWS> struct MassTiles {
    bool by_head;
    int first, last;   // tiles of a query head, or of rows
    int count;         // of all query heads
    __device__ __forceinline__ MassTiles(const AttnArgs &a, const MassSeq &sq, bool heads, int k0, int k1) {
        int i0, i1;
        tokens_that_see(a, sq, k0, k1, i0, i1);
        by_head = heads;
        first = by_head ? i0 / ROWS : (int)((long long)i0 * a.group / ROWS);
        last = i1 > i0 ? (by_head ? (i1 + ROWS - 1) / ROWS : (i1 * a.group + ROWS - 1) / ROWS) : first;
        count = (last - first) * (by_head ? a.group : 1);
    }
};
// Tile u of them: tile `tile` of query head `head` of the key head's.
struct MassAt {
    int head, tile;
    template <int ROWS> __device__ __forceinline__ MassAt(const MassTiles<ROWS> &m, int u) {
        const int each = max(m.last - m.first, 1);
        head = m.by_head ? uniform(u / each) : 0;
        tile = m.first + u - head * each;
    }
    template <int ROWS> __device__ __forceinline__ bool on(const MassTiles<ROWS> &m) {   // says whether the head is another
        if (++tile != m.last || !m.by_head) return false;
        tile = m.first;
        ++head;
        return true;
    }
};

template <typename T, int DP, int KS>
__global__ __launch_bounds__(256, DP * sizeof(T) * KS <= 512 ? 2 : 1) void mass_wide_kernel(MassArgs p) {
    constexpr int QS = DP * (int)sizeof(T) <= 512 ? 2 : 1, ROWS = 32 * QS;   // rows of a tile, in LDS
    using L = AttnTile<T, DP, 4, QS>;
    using Keys = MassKeys<T, DP, KS>;
    using Scores = typename Keys::Scores;
    constexpr int UPR = L::UPR, EU = L::EU, RB = L::RB, KEYS = 128 * KS;
    constexpr int OWN = ROWS / 4, STEP = 64 / UPR;   // rows of a wave's loads, of one
    constexpr float LOG2E = 1.44269504088896340736f;
    extern __shared__ __align__(1024) unsigned char lds[];
    const AttnArgs &a = p.t;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, half = lane >> 5;
    typedef __attribute__((address_space(3))) unsigned char lds_byte;
    const unsigned lds_at = (unsigned)(uintptr_t)(lds_byte *)lds;
    const float c = a.scale_log2;
    if (DP != a.dim)   // the columns past the head, which no load writes
        for (int i = tid; i < 2 * L::SIDE / 16; i += 256) reinterpret_cast<uint4 *>(lds)[i] = make_uint4(0, 0, 0, 0);
    // a sequence's workgroups one after the other, so that a long one's are on all compute units, and of these the ones with the
    // first keys, which the most rows see, first
    const unsigned x1 = div_by(blockIdx.x, p.div_heads), x2 = div_by(x1, p.div_rows), b = div_by(x2, p.div_blocks);
    const int hp = (int)(blockIdx.x - x1 * p.head_parts), rp = (int)(x1 - x2 * p.row_parts), kb0 = (int)(x2 - b * p.blocks);
    // share `part` of `count` things: an even one, the first ones one more
    auto from = [](int count, int part, int parts, const FastDiv &div) __attribute__((always_inline)) {
        const int each = (int)div_by(count, div);
        return each * part + min(part, count - each * parts);
    };
    const int h0 = from(a.kv_heads, hp, p.head_parts, p.div_heads), h1 = from(a.kv_heads, hp + 1, p.head_parts, p.div_heads);
    MassSeq sq(a, (int)b);
    sq.settle();
    const int32_t *list = a.page_list + (long long)b * a.list_stride;
    const int nrows = sq.nq * a.group, past = sq.kv - sq.nq, heads = a.kv_heads * a.group;
    // this lane's loads: row row0 + i * STEP of a tile, its unit that belongs at this lane's place in LDS.  Where a tile's rows are
    // whole tokens' of all query heads, or one head's, they lie at the same distances in every tile, a tile apart.
    const MassOrder<ROWS> order(a, sq);
    const int shift = max(order.shift, 0), few = (1 << shift) - 1, step_tokens = ROWS >> shift;
    const int own = lane / UPR, slot = lane % UPR, row0 = w * OWN + own;
    unsigned unit[L::LOADS], place[L::LOADS];
#pragma unroll
    for (int i = 0; i < L::LOADS; ++i) {
        const int r = row0 + i * STEP;
        unit[i] = slot ^ L::key_unit(r);
        place[i] = (unsigned)(r >> shift) * (unsigned)(a.qs[0] * sizeof(T)) + (unsigned)(r & few) * (unsigned)(a.qs[1] * sizeof(T)) + unit[i] * 16;
    }
    // log-sums 32 rows on (shift 6: a token's heads)
    const unsigned log_step = shift < 6 ? (unsigned)(32 >> shift) * (unsigned)heads : 32;
    const T *q0 = static_cast<const T *>(a.q) + (long long)sq.q0 * a.qs[0];
    const float *lse0 = p.lse + (long long)sq.q0 * heads;

    for (int kb = kb0; (long long)kb * KEYS < sq.kv; kb += p.blocks) {
        const int k0 = kb * KEYS + w * 32 * KS;   // this wave's keys
        const MassTiles<ROWS> tiles(a, sq, order.by_head, kb * KEYS, min(kb * KEYS + KEYS, sq.kv));
        const bool by_head = tiles.by_head;
        const int u0 = uniform(from(tiles.count, rp, p.row_parts, p.div_rows));
        const int u1 = uniform(from(tiles.count, rp + 1, p.row_parts, p.div_rows));
        // tiles that lie within the new tokens; those of them, [whole0, whole1), whose rows see all of this wave's keys (rows
        // past the last count nowhere, their log-sums are infinite)
        const int full = by_head ? sq.nq / ROWS : (order.shift < 0 ? 0 : nrows / ROWS), each = by_head ? 1 : a.group;
        int whole0 = 0, whole1 = k0 + 32 * KS <= sq.kv ? (sq.nq * each + ROWS - 1) / ROWS : 0;
        if (a.causal) whole0 = (min(max(k0 + 32 * KS - 1 - past, 0), sq.nq) * each + ROWS - 1) / ROWS;
        if (a.window > 0) {
            const long long seen = (long long)k0 - past + a.window;   // tokens before this one see the first key
            if (seen < sq.nq) whole1 = min(whole1, max((int)seen, 0) * each / ROWS);
        }
        Keys keys;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int e = 0; e < 16; ++e) keys.got[ks][e] = 0.0f;
#pragma unroll 1
        for (int hk = h0; hk < h1 && u1 > u0; ++hk) {
            const T *q_head = q0 + (long long)hk * a.group * a.qs[1];
            const float *lse_head = lse0 + hk * a.group;
            // row `in` of a tile: its token and its query head among the key head's; past the last one, that one again
            auto row_of = [&](const MassAt &at, int in, int &token, int &head) __attribute__((always_inline)) {
                token = min(ROWS * at.tile + in, by_head ? sq.nq - 1 : nrows - 1);
                head = at.head;
                if (!by_head) {
                    const int r = token;
                    token = (int)div_by(r, a.div_group);
                    head = r - token * a.group;
                }
            };
            // The loop is 32 rows ahead with the scores: those of the next rows go through the matrix cores while the weights
            // of these go through the vector unit.  A tile is read while the next one is on its way, with its rows' log-sums,
            // which are loaded first, so that the wait for the tile is theirs too.
            MassAt here(tiles, u0), coming = here;
            int issued = u0;
            const T *q_at;
            const float *lse_at;
            auto locate = [&]() __attribute__((always_inline)) {
                q_at = q_head + (long long)(step_tokens * coming.tile) * a.qs[0] + (long long)coming.head * a.qs[1];
                lse_at = lse_head + (long long)(step_tokens * coming.tile) * heads + coming.head;
            };
            locate();
            float log[QS], next_log[QS] = {};
            // the next tile's log-sums, and its rows into half `issued - u0` % 2 of LDS
            auto issue = [&]() __attribute__((always_inline)) {
                if (issued < u1) {
                    const unsigned to = lds_at + ((issued - u0) & 1) * L::SIDE + w * OWN * RB;
                    if (p.near && coming.tile < full) {
                        int r = l32;
                        asm volatile("" : "+v"(r));   // here: the offset would not find a register across the loop
                        const unsigned log_at = (unsigned)(r >> shift) * (unsigned)heads + (r & few);
#pragma unroll
                        for (int i = 0; i < QS; ++i) next_log[i] = lse_at[log_at + i * log_step];
#pragma unroll
                        for (int i = 0; i < L::LOADS; ++i) {
                            if (DP != a.dim && (int)unit[i] * EU >= a.dim) continue;
                            load_to_lds(reinterpret_cast<const char *>(q_at), place[i], to + i * 1024);
                        }
                    } else {
                        int token, head;
#pragma unroll
                        for (int i = 0; i < QS; ++i) {
                            row_of(coming, 32 * i + l32, token, head);
                            next_log[i] = lse_head[(long long)token * heads + head];
                            if (ROWS * coming.tile + 32 * i + l32 >= (by_head ? sq.nq : nrows)) next_log[i] = INFINITY;
                        }
#pragma unroll
                        for (int i = 0; i < L::LOADS; ++i) {
                            if (DP != a.dim && (int)unit[i] * EU >= a.dim) continue;
                            row_of(coming, row0 + i * STEP, token, head);
                            const T *from = q_head + (long long)token * a.qs[0] + (long long)head * a.qs[1];
                            load_to_lds(reinterpret_cast<const char *>(from) + unit[i] * 16, to + i * 1024);
                        }
                    }
                }
                ++issued;
                if (coming.on(tiles)) {
                    locate();
                } else {
                    q_at += step_tokens * a.qs[0];
                    lse_at += step_tokens * heads;
                }
            };
            // The tile issued last has landed, and nobody reads the one before it any more.
            auto turn = [&]() __attribute__((always_inline)) {
                wait_loads();
                tile_barrier();
#pragma unroll
                for (int i = 0; i < QS; ++i) log[i] = next_log[i] * LOG2E;   // in powers of two
                issue();
            };
            const unsigned char *rows = lds + l32 * RB;   // of tile u, 32 rows at a time
            unsigned at_tile = 0;
            const int f = L::key_unit(l32);   // (of rows 32 + l32 as well)
            __syncthreads();   // the head before this one has been read
            issue();
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {   // past the last key that one again, which counts nowhere
                const int key = min(k0 + 32 * ks + l32, sq.kv - 1), in = (int)div_by(key, a.div_page);
                const char *row = static_cast<const char *>(a.k) + (long long)hk * a.kb[2] +
                                  page_row(min(max(list[in], 0), a.pages - 1), a.kb[0], key - in * a.page, a.kb[1]);
#pragma unroll
                for (int q = 0; q < Keys::NQ; ++q) {
                    const int u = 2 * q + half;
                    const uint4 k = *reinterpret_cast<const uint4 *>(row + (u * EU < a.dim ? u * 16 : 0));
                    keys.kf[ks][q] = u * EU < a.dim ? k : make_uint4(0, 0, 0, 0);
                }
            }
            turn();
            Scores s0, s1;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)   // the scores of the first rows
#pragma unroll
                for (int e = 0; e < 16; ++e) s0[ks][e] = 0.0f;
#pragma unroll
            for (int q = 0; q < Keys::NQ; ++q)
#pragma unroll
                for (int ks = 0; ks < KS; ++ks)
                    Keys::multiply(s0[ks], keys.kf[ks][q], *reinterpret_cast<const uint4 *>(rows + (((2 * q + half) ^ f) << 4)));
            // A tile: the weights of its rows, and the scores of the rows after them (behind the last tile of what lies there,
            // for nobody).  A place of a row's keys: from + those of the lane, up to span.
            auto tile = [&](auto masked, const unsigned (&from)[QS], const unsigned (&span)[QS]) __attribute__((always_inline)) {
                constexpr bool MASKED = decltype(masked)::value;
                if constexpr (QS == 2) {
                    keys.template step<MASKED>(rows + at_tile + 32 * RB, f, s0, s1, c, log[0], from[0], span[0]);
                    const float second = log[1];
                    at_tile ^= L::SIDE;
                    turn();
                    keys.template step<MASKED>(rows + at_tile, f, s1, s0, c, second, from[1], span[1]);
                } else {
                    const float first = log[0];
                    at_tile ^= L::SIDE;
                    turn();
                    keys.template step<MASKED>(rows + at_tile, f, s0, s1, c, first, from[0], span[0]);
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) s0[ks] = s1[ks];
                }
                here.on(tiles);
            };
            for (int u = u0; u < u1; ++u) {
                unsigned from[QS] = {}, span[QS] = {};
                if (here.tile >= whole0)
                    for (int n = min(whole1 - here.tile, u1 - u); n > 0; --n) {
                        tile(std::false_type{}, from, span);
                        ++u;
                    }
                if (u >= u1) break;
#pragma unroll
                for (int i = 0; i < QS; ++i) {
                    int token, head;
                    row_of(here, 32 * i + l32, token, head);
                    const bool is = ROWS * here.tile + 32 * i + l32 < (by_head ? sq.nq : nrows);
                    const int jhi = is ? min(a.causal ? past + token : sq.kv - 1, sq.kv - 1) : -1;
                    const int jlo = a.window > 0 ? max(past + token - a.window + 1, 0) : 0;
                    // (a row that sees nothing: from a place that no key has)
                    from[i] = jhi < jlo ? 1u << 31 : (unsigned)(k0 + 4 * half - jlo);
                    span[i] = jhi < jlo ? 0u : (unsigned)(jhi - jlo);
                }
                tile(std::true_type{}, from, span);
            }
        }
        const int part = hp * p.row_parts + rp;
        const bool alone = p.head_parts * p.row_parts == 1;
        float *to = alone ? p.mass + b * p.mass_stride : p.part + ((long long)part * a.batch + b) * a.capacity;
        const float sum = keys.sum();
        constexpr int MINE = 16 * KS;   // keys of a lane: now each of so many lanes has one's sum
        const int e = l32 % MINE, j = k0 + 32 * (e / 16) + 8 * (e % 16 / 4) + 4 * half + e % 4;
        if (l32 < MINE && j < sq.kv) to[j] = alone ? to[j] + sum : sum;
    }
}

// The blocks of `keys` keys that some row sees, one sequence after the other, in equal runs, one a workgroup: lengths,
// which only the device knows, may be of any kind.  By whole waves.
struct MassRuns {
    long long first, last;   // blocks of this workgroup
    long long upto;          // blocks up to this lane's sequence, of the first 64
    __device__ static long long scan(const AttnArgs &a, int keys, int b) {
        const int lane = threadIdx.x & 63;
        long long incl = 0;
        if (b < a.batch) {
            const MassSeq sq(a, b);
            incl = sq.nq > 0 ? (sq.kv - sq.first(a) + keys - 1) / keys : 0;
        }
        if (a.capacity <= 1 << 29) {   // 64 sequences' blocks, of 16 keys at least, are fewer than 2^32
            uint32_t x = (uint32_t)incl;
#define FT_SCAN(ctrl, rows) x += __builtin_amdgcn_update_dpp(0, x, ctrl, rows, 0xf, false)
            FT_SCAN(0x111, 0xf);   // row_shr 1, 2, 4, 8
            FT_SCAN(0x112, 0xf);
            FT_SCAN(0x114, 0xf);
            FT_SCAN(0x118, 0xf);
            FT_SCAN(0x142, 0xa);   // the last of rows 0 and 2 to rows 1 and 3, of row 1 to rows 2 and 3
            FT_SCAN(0x143, 0xc);
#undef FT_SCAN
            return x;
        }
#pragma unroll
        for (int x = 1; x < 64; x *= 2) {
            const long long v = __shfl_up(incl, x);
            if (lane >= x) incl += v;
        }
        return incl;
    }
    __device__ MassRuns(const AttnArgs &a, int keys) {
        upto = scan(a, keys, threadIdx.x & 63);
        long long total = __shfl(upto, 63);
        for (int b0 = 64; b0 < a.batch; b0 += 64) total += __shfl(scan(a, keys, b0 + (threadIdx.x & 63)), 63);
        total = uniform(total);
        // (up to 2^55 blocks, 2^10 workgroups)
        first = uniform(divide(total * blockIdx.x, gridDim.x));
        last = uniform(divide(total * (blockIdx.x + 1), gridDim.x));
    }
    // the sequence that block `at` belongs to, and where that sequence's begin
    __device__ int find(const AttnArgs &a, int keys, long long at, long long &base) const {
        base = 0;
        for (int b0 = 0;; b0 += 64) {
            const long long incl = b0 == 0 ? upto : scan(a, keys, b0 + (threadIdx.x & 63));
            const unsigned long long past = __ballot(base + incl > at);
            if (past || b0 + 64 >= a.batch) {
                const int lane = past ? __builtin_ctzll(past) : 63;
                base += lane > 0 ? __shfl(incl, max(lane - 1, 0)) : 0;
                return min(b0 + lane, a.batch - 1);
            }
            base += __shfl(incl, 63);
        }
    }
};

template <typename T, int DP> struct MassFew {
    using S = StreamTile<T, DP>;
    static constexpr int KEYS = S::KEYS, TILES = DP * sizeof(T) <= 512 ? 2 : 1;   // of a wave's loads; in registers
    static constexpr int WAVES = DP * sizeof(T) <= 256 ? 3 : 2;                    // on a SIMD
};
template <typename T, int DP>
__global__ __launch_bounds__(256, (MassFew<T, DP>::WAVES)) void mass_few_kernel(MassArgs p) {
    using L = StreamTile<T, DP>;
    constexpr bool BF = sizeof(T) == 2;
    constexpr int S2 = L::S2, KEYS = L::KEYS, EU = L::EU, NQ = L::NQ, TILES = MassFew<T, DP>::TILES, BLOCK = KEYS * TILES;
    __shared__ float sums[4][BLOCK];
    const AttnArgs &a = p.t;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n16 = lane & 15, h = lane >> 4;
    const float c = a.scale_log2;
    const MassRuns runs(a, KEYS);
    if (runs.first >= runs.last) return;
    long long base;
    int b = uniform(runs.find(a, KEYS, runs.first, base));
    base = uniform(base);
    for (long long at = runs.first; at < runs.last;) {
        MassSeq sq(a, b);
        sq.settle();
        const int lo = sq.first(a), blocks = sq.nq > 0 ? (sq.kv - lo + KEYS - 1) / KEYS : 0;
        if (at >= base + blocks) {   // the run goes on in a later sequence
            base += blocks;
            ++b;
            continue;
        }
        const int k0 = lo + (int)(at - base) * KEYS, some = (int)min((long long)TILES, runs.last - at);
        const int k1 = min(k0 + some * KEYS, sq.kv);
        at += min(some, blocks - (int)(at - base));
        int i0, i1;
        tokens_that_see(a, sq, k0, k1, i0, i1);
        const int r0 = uniform(i0 * a.group / 16), r1 = uniform((i1 * a.group + 15) / 16);   // tiles of 16 rows
        const int32_t *list = a.page_list + (long long)b * a.list_stride;
        static_assert(BLOCK <= 256, "a thread has a key");
        float *to = p.mass + b * p.mass_stride + k0;
        const float before = to[min((int)threadIdx.x, k1 - k0 - 1)];
        const char *krow[TILES][S2];
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int s = 0; s < S2; ++s) {   // past the last key that one again, which counts nowhere
                const int key = min(k0 + t * KEYS + 16 * s + n16, k1 - 1), in = (int)div_by(key, a.div_page);
                krow[t][s] = static_cast<const char *>(a.k) +
                             page_row(min(max(list[in], 0), a.pages - 1), a.kb[0], key - in * a.page, a.kb[1]);
            }
        uint4 kf[TILES][S2][NQ], qf[NQ];
        auto load_k = [&](int t, int hk) __attribute__((always_inline)) {
#pragma unroll
            for (int s = 0; s < S2; ++s)
#pragma unroll
                for (int q = 0; q < NQ; ++q)
                    kf[t][s][q] = *reinterpret_cast<const uint4 *>(krow[t][s] + (long long)hk * a.kb[2] +
                                                                   ((4 * q + h) * EU < a.dim ? (4 * q + h) * 16 : 0));
        };
        float log = 0.0f;
        auto load_q = [&](int hk, int rt, uint4 (&to)[NQ], float &l) __attribute__((always_inline)) {
            const MassRow row(a, sq, hk, rt * 16 + n16);
            const T *from = static_cast<const T *>(a.q) + (long long)(sq.q0 + row.qi) * a.qs[0] + (long long)row.head * a.qs[1];
#pragma unroll
            for (int q = 0; q < NQ; ++q) {
                const int col = (4 * q + h) * EU;
                to[q] = col < a.dim ? *reinterpret_cast<const uint4 *>(from + col) : make_uint4(0, 0, 0, 0);
            }
            l = p.lse[(long long)(sq.q0 + row.qi) * a.kv_heads * a.group + row.head];
        };
        f32x4_t acc[TILES][S2];
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int s = 0; s < S2; ++s) acc[t][s] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
        int hk = w, rt = r0;
        if (hk < a.kv_heads) {
            load_q(hk, rt, qf, log);
#pragma unroll
            for (int t = 0; t < TILES; ++t) load_k(t, hk);
        }
        while (hk < a.kv_heads) {
            const bool same = rt + 1 < r1;   // rows of this key head are left
            const int next_rt = same ? rt + 1 : r0, next_hk = same ? hk : hk + 4;
            const bool more = next_hk < a.kv_heads;
            const MassRow row(a, sq, hk, rt * 16 + n16);
            const int jhi = min(row.jhi, k1 - 1);
            uint4 next_q[NQ];
            float next_log = 0.0f;
            if (more) load_q(next_hk, next_rt, next_q, next_log);
            const float lg = log * 1.44269504088896340736f;
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                if (DP != a.dim) {   // keys' columns past the head: zero, as the queries' are
#pragma unroll
                    for (int s = 0; s < S2; ++s)
#pragma unroll
                        for (int q = 0; q < NQ; ++q)
                            if ((4 * q + h) * EU >= a.dim) kf[t][s][q] = make_uint4(0, 0, 0, 0);
                }
#pragma unroll
                for (int s = 0; s < S2; ++s) {
                    f32x4_t sc = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int q = 0; q < NQ; ++q) {
                        if constexpr (BF) {
                            sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                                __builtin_bit_cast(bf16x8_t, kf[t][s][q]), __builtin_bit_cast(bf16x8_t, qf[q]), sc, 0, 0, 0);
                        } else {
                            const float4 ka = __builtin_bit_cast(float4, kf[t][s][q]), qb = __builtin_bit_cast(float4, qf[q]);
                            sc = __builtin_amdgcn_mfma_f32_16x16x4f32(ka.x, qb.x, sc, 0, 0, 0);
                            sc = __builtin_amdgcn_mfma_f32_16x16x4f32(ka.y, qb.y, sc, 0, 0, 0);
                            sc = __builtin_amdgcn_mfma_f32_16x16x4f32(ka.z, qb.z, sc, 0, 0, 0);
                            sc = __builtin_amdgcn_mfma_f32_16x16x4f32(ka.w, qb.w, sc, 0, 0, 0);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int j = k0 + t * KEYS + 16 * s + 4 * h + i;
                        const float x = fmaf(sc[i], c, -lg);
                        acc[t][s][i] += __builtin_amdgcn_exp2f(j >= row.jlo && j <= jhi ? x : -INFINITY);
                    }
                }
                if (more && !same) load_k(t, next_hk);
            }
#pragma unroll
            for (int q = 0; q < NQ; ++q) qf[q] = next_q[q];
            log = next_log;
            hk = next_hk;
            rt = next_rt;
        }
        __syncthreads();   // the block before this one has been read
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int s = 0; s < S2; ++s)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float v = sum16(acc[t][s][i]);
                    if (n16 == 0) sums[w][t * KEYS + 16 * s + 4 * h + i] = v;
                }
        __syncthreads();
        const int j = threadIdx.x;
        if (j < k1 - k0) to[j] = before + (((sums[0][j] + sums[1][j]) + sums[2][j]) + sums[3][j]);
    }
}

template <typename T, int DP, int KS> hipError_t mass_wide_go(const MassArgs &a, unsigned blocks, hipStream_t st) {
    constexpr int LDS = 2 * AttnTile<T, DP, 4, (DP * sizeof(T) <= 512 ? 2 : 1)>::SIDE;
    auto kernel = mass_wide_kernel<T, DP, KS>;
    if constexpr (LDS > 65536) {
        static std::atomic<uint64_t> raised{0};   // devices whose limit is raised for this kernel
        const hipError_t err = raise_lds_limit(reinterpret_cast<const void *>(kernel), LDS, raised);
        if (err != hipSuccess) return err;
    }
    kernel<<<blocks, 256, LDS, st>>>(a);
    return hipGetLastError();
}
template <typename T, int DP> hipError_t mass_go(const MassPlan &pl, const MassArgs &a, hipStream_t st) {
    if (!pl.wide) {
        mass_few_kernel<T, DP><<<(unsigned)pl.blocks, 256, 0, st>>>(a);
        return hipGetLastError();
    }
    const unsigned blocks = (unsigned)pl.blocks * a.t.batch * pl.head_parts * pl.row_parts;
    if constexpr (DP * sizeof(T) <= 256)
        if (pl.keys == 256) return mass_wide_go<T, DP, 2>(a, blocks, st);
    return mass_wide_go<T, DP, 1>(a, blocks, st);
}
template <typename T> hipError_t mass_pick(const MassPlan &pl, const MassArgs &a, hipStream_t st) {
    if (pl.dp == 64) return mass_go<T, 64>(pl, a, st);
    if (pl.dp == 128) return mass_go<T, 128>(pl, a, st);
    return mass_go<T, 256>(pl, a, st);
}

}  // namespace ftcnn
