// Rows out of a paged cache: of each sequence's n rows the k that come first stay, by (kept for its position,
// larger weight, lower place).  Where k < n, the i-th place below k whose row goes takes the i-th row from k on
// that stays, so that no more rows move than have to, and none that a move reads is written by another.
//
// Which stay: the k-th largest weight comes from counts of the bits of the weights' images as ordered integers, 11, 11 and 10
// at a time, until a whole bin stays; ties go to the lower places, by counts of the waves' votes.  Each wave has a run of
// neighbouring places, so that places in order are waves in order.  What bounds it is the chain of passes and their barriers,
// with next to no work: loops over places in LDS are short code (held in registers they were straight code, 16 us for 64
// sequences of 4097 against 12 now), without branches, and sums over lanes and waves go through DPP.
//
// select_kernel: a workgroup a sequence, which keeps up to 16384 places in LDS.  64 sequences of 4097 rows, one out: 11.5 us.
// part_kernel: five launches for longer ones, a workgroup for every 8192 places: three count bits, each with the limit from
// the counts of the one before in all parts, one counts what moves, one writes.  131072 rows halved: 34 us (49 in parts of
// 16384, 36 in parts of 4096; of 64 sequences of 32768 46, 52 in parts of 4096).
// move_kernel: the moves' rows of all heads, keys and values, 16 bytes a lane, two moves on their way.  The same 131072 rows:
// 61 us, 4.4 TB/s read and written.
#include <algorithm>

#include "evict.h"
#include "paged_attn.h"

namespace ftcnn {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
constexpr int kWaves = kEvictWaves, kSelect = 64 * kWaves;
constexpr int kBins = kEvictBins, kPasses = 3;

// Bits of pass p: 31-21, 20-10, 9-0.
__device__ __forceinline__ int shift_of(int p) { return p == 0 ? 21 : (p == 1 ? 10 : 0); }
__device__ __forceinline__ uint32_t bits_of(int p) { return p == 2 ? 0x3ffu : 0x7ffu; }

// An integer that is in the order of the weight: NaN first, both zeros alike.
__device__ __forceinline__ uint32_t ordered(float w) {
    if (w != w) return 0;
    const uint32_t u = w == 0.0f ? 0u : __float_as_uint(w);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// The sum over the lanes up to this one, of 16 or 64.
template <int LANES> __device__ __forceinline__ uint32_t scan(uint32_t x) {
#define FT_SCAN(ctrl, rows) x += __builtin_amdgcn_update_dpp(0, x, ctrl, rows, 0xf, false)
    FT_SCAN(0x111, 0xf);   // row_shr 1, 2, 4, 8
    FT_SCAN(0x112, 0xf);
    FT_SCAN(0x114, 0xf);
    FT_SCAN(0x118, 0xf);
    if (LANES == 64) {
        FT_SCAN(0x142, 0xa);   // the last of rows 0 and 2 to rows 1 and 3, of row 1 to rows 2 and 3
        FT_SCAN(0x143, 0xc);
    }
#undef FT_SCAN
    return x;
}

// A sequence as the call has it.
struct EvictSeq {
    int n, k, first, since;
    bool no_since;
    const float *mass;
    const int32_t *positions;
    float *mass_out;
    int32_t *positions_out;
    __device__ EvictSeq(const EvictArgs &a, int b) {
        n = min(max(a.kv_lens[b], 0), a.capacity);
        k = min(max(a.keep[b], 0), n);
        first = a.first;
        no_since = !a.since;
        since = a.since ? a.since[b] : 0;
        mass = a.mass + b * a.ms;
        positions = a.positions ? a.positions + b * a.ps : nullptr;
        mass_out = a.mass_out + b * a.mos;
        positions_out = a.positions_out + b * a.pos;
    }
    __device__ __forceinline__ int position(int j) const { return positions ? positions[j] : j; }
    __device__ __forceinline__ bool held_at(int p) const { return (p < first) | (!no_since & (p >= since)); }   // kept for its position
    // what stays where it is
    __device__ __forceinline__ void keep(int j, float m, int p) const {
        if (mass != mass_out) mass_out[j] = m;
        if (positions != positions_out) positions_out[j] = p;
    }
    __device__ __forceinline__ void keep(int j) const { keep(j, mass[j], position(j)); }
    __device__ __forceinline__ void move(int to, int from, float m, int p) const {   // (the outputs may be the inputs)
        mass_out[to] = m;
        positions_out[to] = p;
        clear(from);
    }
    __device__ __forceinline__ void clear(int j) const {
        mass_out[j] = 0.0f;
        positions_out[j] = -1;
    }
};

// The places [p0, p1) of a sequence in a workgroup: this wave's from `base` on, 64 together, `run` of them.  The weights and
// positions of the first of them stay in LDS, each lane's for itself; what there are more, where a sequence is longer than its
// caller said, is read again.  (In registers the loops are straight code, which takes longer to fetch than to run.)
struct Places {
    const float *mass;
    const int32_t *pos;
    int base, run, near, end;
    uint32_t flags = 0;   // bit i of the near ones: kept for its position
    __device__ __forceinline__ Places(const EvictSeq &s, int p0, int p1, float *room, int held) {
        constexpr int AHEAD = 8;
        const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        run = (p1 - p0 + kSelect - 1) / kSelect;
        near = min(run, held / kSelect);
        base = p0 + w * run * 64;
        end = p1;
        float *m_at = room + w * near * 64 + lane;   // (all near: by places)
        int32_t *p_at = reinterpret_cast<int32_t *>(m_at + held);
        mass = m_at;
        pos = p_at;
        for (int i = 0; i < near; i += AHEAD) {   // (of places past the last: that one's, for nobody)
            float m[AHEAD];
            int p[AHEAD];
#pragma unroll
            for (int q = 0; q < AHEAD; ++q) {
                const int j = min(base + 64 * (i + q) + lane, p1 - 1);
                m[q] = s.mass[j];
                p[q] = j;
            }
            if (s.positions) {
#pragma unroll
                for (int q = 0; q < AHEAD; ++q) p[q] = s.positions[p[q]];
            }
#pragma unroll
            for (int q = 0; q < AHEAD; ++q) {
                if (i + q >= near) break;
                m_at[64 * (i + q)] = m[q];
                if (s.positions) p_at[64 * (i + q)] = p[q];
                flags |= (uint32_t)s.held_at(p[q]) << (i + q);
            }
        }
    }
    // f(place, whether it is there, its integer, whether it is kept for its position, its index of the near ones or -1), all
    // lanes together
    template <typename F> __device__ __forceinline__ void each(const EvictSeq &s, F f) const {
        int j = base + (threadIdx.x & 63);
        for (int i = 0; i < near; ++i, j += 64) f(j, j < end, ordered(mass[64 * i]), (flags >> i & 1) != 0, i);
        for (int i = near; i < run; ++i, j += 64) {
            const int at = min(j, end - 1);
            f(j, j < end, ordered(s.mass[at]), s.held_at(s.position(at)), -1);
        }
    }
};

// What the passes found: candidates (those kept for their positions, or the others) whose bits under `mask` are over `limit`
// stay, and of those that equal it the first `need` of `equal`.
struct Limit {
    uint32_t limit = 0, mask = 0, need, equal;
    bool of_held;
    // Those that are kept for their positions all stay, and the rest comes from the others; or they are too many.
    __device__ __forceinline__ Limit(uint32_t k, uint32_t kept) {
        of_held = kept > k;
        need = of_held ? k : k - kept;
        equal = need ? 0xffffffffu : 0;
        if (need == 0) limit = 0xffffffffu;   // none is at it or over it
    }
    __device__ __forceinline__ bool candidate(bool in, bool held) const { return in & (held == of_held); }
    __device__ __forceinline__ bool tie(bool in, uint32_t x, bool held) const { return candidate(in, held) & ((x & mask) == limit); }
    __device__ __forceinline__ bool open() const { return need < equal; }   // some of the equal ones stay, and some go
};

// The sum over the workgroup's waves of what each has; before: of the waves before this one.
__device__ __forceinline__ uint32_t sum_waves(uint32_t mine, uint32_t *room, uint32_t &before) {
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (lane == 0) room[w] = mine;
    __syncthreads();
    const uint32_t sums = scan<16>(room[lane % kWaves]);
    before = w ? __builtin_amdgcn_readlane(sums, w - 1) : 0;
    return __builtin_amdgcn_readlane(sums, kWaves - 1);
}

// Two of them with one barrier: the sums, and `before` of each.
__device__ __forceinline__ uint2 sum_waves(uint2 mine, uint32_t *room0, uint32_t *room1, uint2 &before) {
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (lane == 0) room1[w] = mine.y;
    const uint32_t x = sum_waves(mine.x, room0, before.x), sums = scan<16>(room1[lane % kWaves]);
    before.y = w ? __builtin_amdgcn_readlane(sums, w - 1) : 0;
    return make_uint2(x, __builtin_amdgcn_readlane(sums, kWaves - 1));
}

// The highest bin with `need` candidates in it and those above it, of counts c0, c1 of bins kBins - 1 - 2 tid and the one below
// it: narrows the limit to that bin.  room: kWaves + 3 words.
__device__ __forceinline__ void narrow(Limit &l, uint32_t c0, uint32_t c1, int pass, uint32_t *room) {
    const int tid = threadIdx.x;
    uint32_t before;
    uint32_t incl = scan<64>(c0 + c1);
    sum_waves(__builtin_amdgcn_readlane(incl, 63), room, before);
    incl += before;
    const uint32_t below = incl - c0 - c1;
    if (below < l.need && l.need <= incl) {
        const bool second = l.need > below + c0;
        room[kWaves] = kBins - 1 - 2 * tid - (second ? 1 : 0);
        room[kWaves + 1] = below + (second ? c0 : 0);
        room[kWaves + 2] = second ? c1 : c0;
    }
    __syncthreads();
    l.limit |= room[kWaves] << shift_of(pass);
    l.mask |= bits_of(pass) << shift_of(pass);
    l.need -= room[kWaves + 1];
    l.equal = room[kWaves + 2];
}

// The candidates whose bits so far are the limit's, counted by the bits of a pass.
__device__ __forceinline__ void count_bits(const EvictSeq &s, const Places &places, const Limit &l, int pass, uint32_t *bins) {
    const int at = shift_of(pass);
    const uint32_t bits = bits_of(pass);
    places.each(s, [&](int, bool in, uint32_t x, bool held, int) {
        if (l.tie(in, x, held)) atomicAdd(&bins[x >> at & bits], 1u);
    });
}
__device__ __forceinline__ uint32_t count_held(const EvictSeq &s, const Places &places) {
    uint32_t mine = 0;
    places.each(s, [&](int, bool in, uint32_t, bool held, int) { mine += __popcll(__builtin_amdgcn_ballot_w64(in & held)); });
    return mine;
}
__device__ __forceinline__ uint32_t count_ties(const EvictSeq &s, const Places &places, const Limit &l) {
    uint32_t mine = 0;
    places.each(s, [&](int, bool in, uint32_t x, bool held, int) { mine += __popcll(__builtin_amdgcn_ballot_w64(l.tie(in, x, held))); });
    return mine;
}

// The set lanes of m below this one.
__device__ __forceinline__ uint32_t below(unsigned long long m) {
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0));
}
// Calls f(place, whether it stays, whether it is there and goes, its index of the near ones or -1), this wave's ties ranked from
// `rank` on.
template <typename F>
__device__ __forceinline__ void each_stay(const EvictSeq &s, const Places &places, const Limit &l, uint32_t rank, F f) {
    places.each(s, [&](int j, bool in, uint32_t x, bool held, int i) {
        bool tie = l.tie(in, x, held);
        const bool over = l.candidate(in, held) & ((x & l.mask) > l.limit);
        if (l.open()) {
            const unsigned long long vote = __builtin_amdgcn_ballot_w64(tie);
            tie = tie & (rank + below(vote) < l.need);
            rank += __popcll(vote);
        }
        const bool stays = over | tie | (in & held & !l.of_held);
        f(j, stays, in & !stays, i);
    });
}
// The holes below k and the rows from k on that stay, of this wave.
__device__ __forceinline__ void count_moves(const EvictSeq &s, const Places &places, const Limit &l, uint32_t rank, uint32_t &holes,
                                            uint32_t &late) {
    holes = late = 0;
    each_stay(s, places, l, rank, [&](int j, bool stays, bool goes, int) {
        holes += __popcll(__builtin_amdgcn_ballot_w64(goes & (j < s.k)));
        late += __popcll(__builtin_amdgcn_ballot_w64(stays & (j >= s.k)));
    });
}
// Writes them to the lists, from hole_at and late_at on, and to the outputs what stays where it is and what is free from k on.
// near: to lists in LDS as well (to, from by turns).
__device__ __forceinline__ void write_moves(const EvictSeq &s, const Places &places, const Limit &l, uint32_t rank, uint32_t hole_at,
                                            uint32_t late_at, int32_t *to, int32_t *from, uint16_t *near) {
    each_stay(s, places, l, rank, [&](int j, bool stays, bool goes, int i) {
        const bool low = j < s.k, hole = goes & low, moving = stays & !low;
        const unsigned long long h = __builtin_amdgcn_ballot_w64(hole), m = __builtin_amdgcn_ballot_w64(moving);
        if (hole) {
            to[hole_at + below(h)] = j;
            if (near) near[2 * (hole_at + below(h))] = (uint16_t)j;
        }
        if (moving) {
            from[late_at + below(m)] = j;
            if (near) near[2 * (late_at + below(m)) + 1] = (uint16_t)j;
        }
        hole_at += __popcll(h);
        late_at += __popcll(m);
        if (stays & low) {
            if (i >= 0) s.keep(j, places.mass[64 * i], s.positions ? places.pos[64 * i] : j);
            else s.keep(j);
        }
        if (goes & !low) s.clear(j);
    });
}

__global__ __launch_bounds__(kSelect) void select_kernel(EvictArgs a) {
    extern __shared__ float held[];
    __shared__ uint32_t bins[kPasses][kBins];
    __shared__ uint32_t room[7][kWaves + 3];
    const int b = blockIdx.x, tid = threadIdx.x;
    const EvictSeq s(a, b);
    const int n = s.n, k = s.k;
    int moves = 0;
    if (k > 0 && k < n) {
        for (int i = tid; i < kPasses * kBins; i += kSelect) bins[0][i] = 0;
        const Places places(s, 0, n, held, a.held);
        uint32_t before;
        Limit l(k, sum_waves(count_held(s, places), room[0], before));
        for (int pass = 0; pass < kPasses && l.open(); ++pass) {   // until the whole bin stays
            count_bits(s, places, l, pass, bins[pass]);
            __syncthreads();
            narrow(l, bins[pass][kBins - 1 - 2 * tid], bins[pass][kBins - 2 - 2 * tid], pass, room[1 + pass]);
        }
        uint32_t rank = 0;   // of the next tie of this wave
        if (l.open()) sum_waves(count_ties(s, places, l), room[4], rank);
        uint2 mine, at;      // holes and rows that move
        count_moves(s, places, l, rank, mine.x, mine.y);
        moves = (int)sum_waves(mine, room[5], room[6], at).x;
        int32_t *to = a.to + b * a.half, *from = a.from + b * a.half;
        // the lists in LDS, where the bins were, save the way to memory and back
        if (places.near == places.run && moves <= kPasses * kBins) {
            uint16_t *list = reinterpret_cast<uint16_t *>(bins[0]);
            write_moves(s, places, l, rank, at.x, at.y, to, from, list);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            tile_barrier();
            const float *held_mass = held;
            const int32_t *held_at = reinterpret_cast<const int32_t *>(held + a.held);
            for (int i = tid; i < moves; i += kSelect) {
                const int t = list[2 * i], f = list[2 * i + 1];
                s.move(t, f, held_mass[f], s.positions ? held_at[f] : f);
            }
        } else {
            write_moves(s, places, l, rank, at.x, at.y, to, from, nullptr);
            __syncthreads();
            for (int i = tid; i < moves; i += kSelect) s.move(to[i], from[i], s.mass[from[i]], s.position(from[i]));
        }
    } else {
        for (int j = tid; j < n; j += kSelect) {
            if (j < k) s.keep(j);
            else s.clear(j);
        }
        __syncthreads();   // the length, which may be written where it was, has been read
    }
    if (tid == 0) {
        a.lens_out[b] = k;
        a.counts[b] = moves;
    }
    for (int j = n + tid; j < a.capacity; j += kSelect) s.clear(j);
}

// The sum of f over the first n parts, by each wave for itself.
template <typename F> __device__ __forceinline__ uint32_t over_parts(int n, F f) {
    uint32_t sum = 0;
    for (int i = threadIdx.x & 63; i < n; i += 64) sum += f(i);
    return __builtin_amdgcn_readlane(scan<64>(sum), 63);
}

// A launch of five for the parts of sequences.  0 to 2 count the bits of that pass, 3 what moves, 4 writes.
template <int STEP> __global__ __launch_bounds__(kSelect) void part_kernel(EvictArgs a) {
    extern __shared__ float held[];
    __shared__ uint32_t bins[STEP == 0 ? 2 : 1][kBins];
    __shared__ uint32_t room[7][kWaves + 3];
    const int b = (int)(blockIdx.x / (unsigned)a.parts), part = (int)(blockIdx.x % (unsigned)a.parts), tid = threadIdx.x;
    const EvictSeq s(a, b);
    const int p0 = part * kEvictPart, p1 = min(kEvictPart, s.n - p0) + p0;
    const bool choose = s.k > 0 && s.k < s.n;   // or all stay, or none
    if constexpr (STEP == 4) {
        const int last = min(kEvictPart, a.capacity - p0) + p0;
        for (int j = p0 + tid; j < last; j += kSelect) {
            if (j >= s.n) s.clear(j);
            else if (!choose && j < s.k) s.keep(j);
            else if (!choose) s.clear(j);
        }
        if (!choose && part == 0 && tid == 0) a.counts[b] = 0;
    }
    if (!choose || p0 >= s.n) return;
    EvictPart *parts = a.part + (long long)b * a.parts, &mine = parts[part];
    const int used = (s.n - 1) / kEvictPart + 1;
    if (STEP < kPasses)
        for (int i = tid; i < (STEP == 0 ? 2 : 1) * kBins; i += kSelect) bins[0][i] = 0;
    const Places places(s, p0, p1, held, a.held);
    if constexpr (STEP == 0) {   // of both kinds, as it is not known yet from which one is chosen
        uint32_t before;
        const uint32_t kept = sum_waves(count_held(s, places), room[0], before);
        places.each(s, [&](int, bool in, uint32_t x, bool held, int) {
            if (in) atomicAdd(&bins[held ? 1 : 0][x >> shift_of(0)], 1u);
        });
        __syncthreads();
        if (tid == 0) mine.kept = kept;
        for (int i = tid; i < kBins; i += kSelect) {
            mine.bins[0][i] = bins[0][i];
            mine.bins[kPasses][i] = bins[1][i];
        }
    } else {
        Limit l(s.k, over_parts(used, [&](int i) { return parts[i].kept; }));
        if (STEP > 1) {   // after the passes before the last one
            const uint4 f = parts[0].found[STEP - 2];
            l.limit = f.x;
            l.mask = f.y;
            l.need = f.z;
            l.equal = f.w;
        }
        if (STEP <= kPasses && l.open()) {
            constexpr int PASS = STEP - 1;
            const uint32_t *from = parts[0].bins[PASS == 0 && l.of_held ? kPasses : PASS] + kBins - 2 - 2 * tid;
            uint32_t c0 = 0, c1 = 0;
            for (int i = 0; i < used; i += 8) {
                uint2 c[8];
#pragma unroll
                for (int q = 0; q < 8; ++q)
                    c[q] = *reinterpret_cast<const uint2 *>(from + (long long)min(i + q, used - 1) * (sizeof(EvictPart) / 4));
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    c0 += i + q < used ? c[q].y : 0;
                    c1 += i + q < used ? c[q].x : 0;
                }
            }
            narrow(l, c0, c1, PASS, room[1]);
        }
        if (STEP <= kPasses && part == 0 && tid == 0) mine.found[STEP - 1] = make_uint4(l.limit, l.mask, l.need, l.equal);
        if constexpr (STEP < kPasses) {
            if (!l.open()) return;   // no further pass is needed
            __syncthreads();
            count_bits(s, places, l, STEP, bins[0]);
            __syncthreads();
            for (int i = tid; i < kBins; i += kSelect) mine.bins[STEP][i] = bins[0][i];
        } else {
            const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
            if constexpr (STEP == 3) {
                uint32_t rank = 0, holes, late;   // rank: of the next tie of this wave
                if (l.open()) {
                    sum_waves(count_ties(s, places, l), room[4], rank);
                    rank += over_parts(part, [&](int i) { return parts[i].bins[kPasses - 1][l.limit & bits_of(kPasses - 1)]; });
                }
                count_moves(s, places, l, rank, holes, late);
                uint2 at;
                const uint2 sums = sum_waves(make_uint2(holes, late), room[5], room[6], at);
                if (tid == 0) {
                    mine.holes = sums.x;
                    mine.late = sums.y;
                }
                if ((tid & 63) == 0) {
                    mine.hole_at[w] = at.x;
                    mine.late_at[w] = at.y;
                    mine.rank[w] = rank;
                }
            } else {
                const uint32_t hole_at = mine.hole_at[w] + over_parts(part, [&](int i) { return parts[i].holes; });
                const uint32_t late_at = mine.late_at[w] + over_parts(part, [&](int i) { return parts[i].late; });
                const uint32_t moves = over_parts(used, [&](int i) { return parts[i].holes; });
                if (part == 0 && tid == 0) a.counts[b] = (int)moves;
                write_moves(s, places, l, mine.rank[w], hole_at, late_at, a.to + b * a.half, a.from + b * a.half, nullptr);
            }
        }
    }
}

__global__ __launch_bounds__(kThreads) void move_kernel(EvictArgs a) {
    constexpr int AHEAD = 2;   // moves on their way (64 sequences of 4097, a move each: 4.2 us; four on their way 5.6, one 4.1, but 131072
                               // rows halved 66 where two take 61)
    const int b = (int)(blockIdx.x / (unsigned)a.shares), share = (int)(blockIdx.x % (unsigned)a.shares);
    const int moves = a.counts[b];
    if (a.parts) {   // the weights and positions that move, and the length, which nobody else reads here
        const EvictSeq s(a, b);
        for (int i = share * kThreads + threadIdx.x; i < moves; i += a.shares * kThreads) {
            const int f = a.from[b * a.half + i];
            s.move(a.to[b * a.half + i], f, s.mass[f], s.position(f));
        }
        if (share == 0 && threadIdx.x == 0) a.lens_out[b] = s.k;
    }
    const int side = a.kv_heads * a.units, units = 2 * side;   // of a move
    const int together = max(1, kThreads / units);             // moves of a workgroup at a time
    const int sub = together > 1 ? threadIdx.x / units : 0;
    if (sub >= together) return;
    const int32_t *list = a.page_list + b * a.list_stride, *from = a.from + b * a.half, *to = a.to + b * a.half;
    const int step = a.shares * together;
    for (int u = threadIdx.x - sub * units; u < units; u += kThreads) {
        const bool value = u >= side;
        const int x = value ? u - side : u, head = x / a.units, unit = x - head * a.units;
        char *cache = static_cast<char *>(value ? a.v : a.k);
        const unsigned pb = value ? a.vb[0] : a.kb[0], rb = value ? a.vb[1] : a.kb[1];
        cache += (long long)head * (value ? a.vb[2] : a.kb[2]) + unit * 16;
        auto row = [&](int j) {
            const int in = (int)div_by(j, a.div_page), pg = min(max(list[in], 0), a.pages - 1);
            return cache + (unsigned long long)(unsigned)pg * pb + (unsigned long long)(unsigned)(j - in * a.page) * rb;
        };
        for (int i = share * together + sub; i < moves; i += AHEAD * step) {
            u32x4 v[AHEAD];   // (past the last move: that one's, for nobody)
            const char *at[AHEAD];
            char *into[AHEAD];
#pragma unroll
            for (int q = 0; q < AHEAD; ++q) {
                at[q] = row(from[min(i + q * step, moves - 1)]);
                into[q] = row(to[min(i + q * step, moves - 1)]);
            }
#pragma unroll
            for (int q = 0; q < AHEAD; ++q) v[q] = *reinterpret_cast<const u32x4 *>(at[q]);
#pragma unroll
            for (int q = 0; q < AHEAD; ++q)
                if (i + q * step < moves) *reinterpret_cast<u32x4 *>(into[q]) = v[q];
        }
    }
}

}  // namespace

hipError_t launch_evict(const EvictArgs &a, hipStream_t st) {
    const size_t room = (size_t)a.held * (a.positions ? 8 : 4);
    hipError_t err = hipSuccess;
    auto launch = [&](auto which, unsigned groups) {   // the kernel of step `which`, or the one for whole sequences
        if (err != hipSuccess) return;
        constexpr int STEP = decltype(which)::value;
        void (*kernel)(EvictArgs);
        if constexpr (STEP < 0) kernel = select_kernel;
        else kernel = part_kernel<STEP>;
        static std::atomic<uint64_t> raised{0};   // devices whose limit is raised for this kernel
        err = raise_lds_limit(reinterpret_cast<const void *>(kernel), (STEP < 0 ? kEvictHeld : kEvictPart) * 8, raised);
        if (err != hipSuccess) return;
        kernel<<<groups, kSelect, room, st>>>(a);
        err = hipGetLastError();
    };
    if (a.parts) {
        const unsigned groups = (unsigned)a.batch * a.parts;
        launch(std::integral_constant<int, 0>{}, groups);
        launch(std::integral_constant<int, 1>{}, groups);
        launch(std::integral_constant<int, 2>{}, groups);
        launch(std::integral_constant<int, 3>{}, groups);
        launch(std::integral_constant<int, 4>{}, groups);
    } else {
        launch(std::integral_constant<int, -1>{}, (unsigned)a.batch);
    }
    if (err != hipSuccess) return err;
    move_kernel<<<(unsigned)a.batch * a.shares, kThreads, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace ftcnn
