// Rows out of a paged cache: of each sequence's n rows the k that come first stay, by (kept for its position,
// larger weight, lower place).  Where k < n, the i-th place below k whose row goes takes the i-th row from k on
// that stays, so that no more rows move than have to, and none that a move reads is written by another.
//
// Which stay: the k-th largest weight comes from counts of the bits of the weights' images as ordered integers, 11, 11 and 10
// at a time; ties go to the lower places, by counts of the waves' votes.  Each wave has a run of neighbouring places, so that
// places in order are waves in order.  select_kernel: a workgroup a sequence, which holds up to 16384 weights in registers.
// part_kernel: the same in five launches, for long sequences, a workgroup for every 16384 places: three that count bits (each
// adds up what those before counted in all parts), one that counts what each part moves, one that writes.
// move_kernel: the moves' rows of all heads, keys and values, 16 bytes a lane.
#include <algorithm>

#include "evict.h"

namespace ftcnn {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
constexpr int kSelect = 1024, kWaves = kSelect / 64;
constexpr int kHeld = kEvictPart / kSelect;     // weights that a lane keeps in registers
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
    __device__ __forceinline__ bool held(int j) const {   // kept for its position
        const int p = position(j);
        return p < first || (!no_since && p >= since);
    }
    // what stays where it is
    __device__ __forceinline__ void keep(int j) const {
        if (mass != mass_out) mass_out[j] = mass[j];
        if (positions != positions_out) positions_out[j] = position(j);
    }
    __device__ __forceinline__ void move(int to, int from) const {   // (the outputs may be the inputs)
        mass_out[to] = mass[from];
        positions_out[to] = position(from);
        clear(from);
    }
    __device__ __forceinline__ void clear(int j) const {
        mass_out[j] = 0.0f;
        positions_out[j] = -1;
    }
};

// The places [p0, p1) of a sequence in a workgroup: this wave's from `base` on, 64 together, run of them; the first kHeld of a
// lane's in registers.
struct Places {
    int base, run, end;
    uint32_t key[kHeld], flags;   // bit i: kept for its position
    __device__ __forceinline__ Places(const EvictSeq &s, int p0, int p1) {
        const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        run = (p1 - p0 + kSelect - 1) / kSelect;
        base = p0 + w * run * 64;
        end = p1;
        float m[kHeld];
        int p[kHeld];
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {   // (of places past the last: that one's, for nobody)
            if (i >= run) break;
            const int j = min(base + 64 * i + lane, p1 - 1);
            m[i] = s.mass[j];
            p[i] = s.position(j);
        }
        flags = 0;
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            key[i] = 0;
            if (i >= run) continue;
            key[i] = ordered(m[i]);
            flags |= (uint32_t)(p[i] < s.first || (!s.no_since && p[i] >= s.since)) << i;
        }
    }
    // f(place, whether it is there, its integer, whether it is kept for its position), all lanes together
    template <typename F> __device__ __forceinline__ void each(const EvictSeq &s, F f) const {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int i = 0; i < kHeld; ++i)
            if (i < run) {
                const int j = base + 64 * i + lane;
                f(j, j < end, key[i], (flags >> i & 1) != 0);
            }
        for (int i = kHeld; i < run; ++i) {
            const int j = base + 64 * i + lane;
            const bool in = j < end;
            f(j, in, in ? ordered(s.mass[j]) : 0u, in && s.held(j));
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
    }
    __device__ __forceinline__ bool tie(bool in, uint32_t x, bool held) const {
        return in && held == of_held && need > 0 && (x & mask) == limit;
    }
    // rank: of a tie among all
    __device__ __forceinline__ bool stays(bool in, uint32_t x, bool held, bool tie, uint32_t rank) const {
        if (!in || held != of_held) return in && held;
        return need > 0 && ((x & mask) > limit || (tie && rank < need));
    }
};

// The sum over the workgroup's waves of what each has; before: of the waves before this one.
__device__ __forceinline__ uint32_t sum_waves(uint32_t mine, uint32_t *room, uint32_t &before) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    if (lane == 0) room[w] = mine;
    __syncthreads();
    uint32_t sum = 0;
    before = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
        if (i == w) before = sum;
        sum += room[i];
    }
    return sum;
}

// The highest bin with `need` candidates in it and those above it, of counts c0, c1 of bins kBins - 1 - 2 tid and the one below
// it: narrows the limit to that bin.  room: kWaves + 3 words.
__device__ __forceinline__ void narrow(Limit &l, uint32_t c0, uint32_t c1, int pass, uint32_t *room) {
    const int tid = threadIdx.x, lane = tid & 63;
    uint32_t incl = c0 + c1, before;
#pragma unroll
    for (int x = 1; x < 64; x *= 2) {
        const uint32_t v = __shfl_up(incl, x);
        if (lane >= x) incl += v;
    }
    sum_waves(__shfl(incl, 63), room, before);
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
    places.each(s, [&](int, bool in, uint32_t x, bool held) {
        if (in && held == l.of_held && (x & l.mask) == l.limit) atomicAdd(&bins[x >> at & bits], 1u);
    });
}

// Calls f(place, whether it is there, whether it stays) with this wave's ties ranked from `rank` on.
template <typename F>
__device__ __forceinline__ void each_stay(const EvictSeq &s, const Places &places, const Limit &l, uint32_t rank, F f) {
    const unsigned long long lower = (1ull << (threadIdx.x & 63)) - 1;
    places.each(s, [&](int j, bool in, uint32_t x, bool held) {
        const bool tie = l.tie(in, x, held);
        const unsigned long long vote = __ballot(tie);
        f(j, in, l.stays(in, x, held, tie, rank + __popcll(vote & lower)));
        rank += __popcll(vote);
    });
}
__device__ __forceinline__ uint32_t ties_of(const EvictSeq &s, const Places &places, const Limit &l) {
    uint32_t mine = 0;
    places.each(s, [&](int, bool in, uint32_t x, bool held) { mine += __popcll(__ballot(l.tie(in, x, held))); });
    return mine;
}
// The holes below k and the rows from k on that stay, of this wave.
__device__ __forceinline__ void count_moves(const EvictSeq &s, const Places &places, const Limit &l, uint32_t rank, uint32_t &holes,
                                            uint32_t &late) {
    holes = late = 0;
    each_stay(s, places, l, rank, [&](int j, bool in, bool stays) {
        holes += __popcll(__ballot(in && !stays && j < s.k));
        late += __popcll(__ballot(stays && j >= s.k));
    });
}
// Writes them to the lists, from hole_at and late_at on, and to the outputs what stays where it is and what is free from k on.
__device__ __forceinline__ void write_moves(const EvictSeq &s, const Places &places, const Limit &l, uint32_t rank, uint32_t hole_at,
                                            uint32_t late_at, int32_t *to, int32_t *from) {
    const unsigned long long lower = (1ull << (threadIdx.x & 63)) - 1;
    each_stay(s, places, l, rank, [&](int j, bool in, bool stays) {
        const bool hole = in && !stays && j < s.k, moving = stays && j >= s.k;
        const unsigned long long h = __ballot(hole), m = __ballot(moving);
        if (hole) to[hole_at + __popcll(h & lower)] = j;
        if (moving) from[late_at + __popcll(m & lower)] = j;
        hole_at += __popcll(h);
        late_at += __popcll(m);
        if (stays && j < s.k) s.keep(j);
        if (in && !stays && j >= s.k) s.clear(j);
    });
}

__global__ __launch_bounds__(kSelect) void select_kernel(EvictArgs a) {
    __shared__ uint32_t bins[kPasses][kBins];
    __shared__ uint32_t room[7][kWaves + 3];
    const int b = blockIdx.x, tid = threadIdx.x;
    const EvictSeq s(a, b);
    const int n = s.n, k = s.k;
    int moves = 0;
    if (k > 0 && k < n) {
        for (int i = tid; i < kPasses * kBins; i += kSelect) bins[0][i] = 0;
        const Places places(s, 0, n);
        uint32_t kept = 0, before;
        places.each(s, [&](int, bool in, uint32_t, bool held) { kept += __popcll(__ballot(in && held)); });
        Limit l(k, sum_waves(kept, room[0], before));
        for (int pass = 0; pass < kPasses && l.need < l.equal; ++pass) {   // until the whole bin stays
            count_bits(s, places, l, pass, bins[pass]);
            __syncthreads();
            narrow(l, bins[pass][kBins - 1 - 2 * tid], bins[pass][kBins - 2 - 2 * tid], pass, room[1 + pass]);
        }
        uint32_t rank = 0, holes, late, hole_at, late_at;   // rank: of the next tie of this wave
        if (l.need < l.equal) sum_waves(ties_of(s, places, l), room[4], rank);
        count_moves(s, places, l, rank, holes, late);
        moves = (int)sum_waves(holes, room[5], hole_at);
        sum_waves(late, room[6], late_at);
        int32_t *to = a.to + b * a.half, *from = a.from + b * a.half;
        write_moves(s, places, l, rank, hole_at, late_at, to, from);
        __syncthreads();
        for (int i = tid; i < moves; i += kSelect) s.move(to[i], from[i]);
    } else {
        for (int j = tid; j < n; j += kSelect) {
            if (j < k) s.keep(j);
            else s.clear(j);
        }
    }
    __syncthreads();   // the length, which may be written where it was, has been read
    if (tid == 0) {
        a.lens_out[b] = k;
        a.counts[b] = moves;
    }
    for (int j = n + tid; j < a.capacity; j += kSelect) s.clear(j);
}

// A launch of five for the parts of sequences.  0 to 2 count the bits of that pass, 3 what moves, 4 writes.
template <int STEP> __global__ __launch_bounds__(kSelect) void part_kernel(EvictArgs a) {
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
    const Places places(s, p0, p1);
    if constexpr (STEP == 0) {   // of both kinds, as it is not known yet from which one is chosen
        uint32_t kept = 0, before;
        places.each(s, [&](int, bool in, uint32_t, bool held) { kept += __popcll(__ballot(in && held)); });
        kept = sum_waves(kept, room[0], before);
        places.each(s, [&](int, bool in, uint32_t x, bool held) {
            if (in) atomicAdd(&bins[held ? 1 : 0][x >> shift_of(0)], 1u);
        });
        __syncthreads();
        if (tid == 0) mine.kept = kept;
        for (int i = tid; i < kBins; i += kSelect) {
            mine.bins[0][i] = bins[0][i];
            mine.bins[kPasses][i] = bins[1][i];
        }
    } else {
        uint32_t kept = 0;
        for (int i = 0; i < used; ++i) kept += parts[i].kept;
        Limit l(s.k, kept);
        for (int pass = 0; pass < min(STEP, kPasses) && l.need < l.equal; ++pass) {
            const int of = pass == 0 && l.of_held ? kPasses : pass;
            uint32_t c0 = 0, c1 = 0;
            for (int i = 0; i < used; ++i) {
                const uint2 c = *reinterpret_cast<const uint2 *>(&parts[i].bins[of][kBins - 2 - 2 * tid]);
                c0 += c.y;
                c1 += c.x;
            }
            narrow(l, c0, c1, pass, room[1 + pass]);
        }
        if constexpr (STEP < kPasses) {
            if (l.need == l.equal) return;   // no further pass is needed
            __syncthreads();
            count_bits(s, places, l, STEP, bins[0]);
            __syncthreads();
            for (int i = tid; i < kBins; i += kSelect) mine.bins[STEP][i] = bins[0][i];
        } else {
            uint32_t rank = 0, holes, late, hole_at, late_at;   // rank: of the next tie of this wave
            if (l.need < l.equal) {
                sum_waves(ties_of(s, places, l), room[4], rank);
                for (int i = 0; i < part; ++i) rank += parts[i].bins[kPasses - 1][l.limit & bits_of(kPasses - 1)];
            }
            count_moves(s, places, l, rank, holes, late);
            const uint32_t hole_sum = sum_waves(holes, room[5], hole_at), late_sum = sum_waves(late, room[6], late_at);
            if constexpr (STEP == 3) {
                if (tid == 0) {
                    mine.holes = hole_sum;
                    mine.late = late_sum;
                }
            } else {
                uint32_t moves = 0;
                for (int i = 0; i < used; ++i) {
                    hole_at += i < part ? parts[i].holes : 0;
                    late_at += i < part ? parts[i].late : 0;
                    moves += parts[i].holes;
                }
                if (part == 0 && tid == 0) a.counts[b] = (int)moves;
                write_moves(s, places, l, rank, hole_at, late_at, a.to + b * a.half, a.from + b * a.half);
            }
        }
    }
}

__global__ __launch_bounds__(kThreads) void move_kernel(EvictArgs a) {
    constexpr int AHEAD = 4;   // moves on their way
    const int b = (int)(blockIdx.x / (unsigned)a.shares), share = (int)(blockIdx.x % (unsigned)a.shares);
    const int moves = a.counts[b];
    if (a.parts) {   // the weights and positions that move, and the length, which nobody else reads here
        const EvictSeq s(a, b);
        for (int i = share * kThreads + threadIdx.x; i < moves; i += a.shares * kThreads) s.move(a.to[b * a.half + i], a.from[b * a.half + i]);
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
    if (a.parts) {
        const unsigned groups = (unsigned)a.batch * a.parts;
        part_kernel<0><<<groups, kSelect, 0, st>>>(a);
        part_kernel<1><<<groups, kSelect, 0, st>>>(a);
        part_kernel<2><<<groups, kSelect, 0, st>>>(a);
        part_kernel<3><<<groups, kSelect, 0, st>>>(a);
        part_kernel<4><<<groups, kSelect, 0, st>>>(a);
    } else {
        select_kernel<<<(unsigned)a.batch, kSelect, 0, st>>>(a);
    }
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    move_kernel<<<(unsigned)a.batch * a.shares, kThreads, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace ftcnn
