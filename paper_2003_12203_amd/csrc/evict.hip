// Rows out of a paged cache: of each sequence's n rows the k that come first stay, by (kept for its position,
// larger weight, lower place).  Where k < n, the i-th place below k whose row goes takes the i-th row from k on
// that stays, so that no more rows move than have to, and none that a move reads is written by another.
//
// select_kernel: a workgroup a sequence.  The k-th largest weight comes from counts of the bits of the weights' images
// as ordered integers, 11, 11 and 10 at a time; ties go to the lower places, by counts of the waves' votes.  Each wave has a
// run of neighbouring places, so that places in order are waves in order.
// move_kernel: the moves' rows of all heads, keys and values, 16 bytes a lane.
#include <algorithm>

#include "evict.h"

namespace ftcnn {
namespace {

constexpr int kSelect = 1024, kWaves = kSelect / 64;
constexpr int kHeld = 16;     // weights that a lane keeps in registers; further ones are read again
constexpr int kBins = 2048;

// An integer that is in the order of the weight: NaN first, both zeros alike.
__device__ __forceinline__ uint32_t ordered(float w) {
    if (w != w) return 0;
    const uint32_t u = w == 0.0f ? 0u : __float_as_uint(w);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__global__ __launch_bounds__(kSelect) void select_kernel(EvictArgs a) {
    __shared__ uint32_t bins[kBins];
    __shared__ uint32_t wave_sum[kWaves], wave_two[kWaves];
    __shared__ uint32_t found_bin, found_above, found_count;
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = min(max(a.kv_lens[b], 0), a.capacity), k = min(max(a.keep[b], 0), n);
    const float *mass = a.mass + b * a.ms;
    const int32_t *positions = a.positions ? a.positions + b * a.ps : nullptr;
    float *mass_out = a.mass_out + b * a.mos;
    int32_t *positions_out = a.positions_out + b * a.pos;
    const bool moved_mass = mass != mass_out, moved_positions = positions != positions_out;
    const int since = a.since ? a.since[b] : INT32_MAX;
    const bool all = !a.since;   // no position is late
    auto position = [&](int j) { return positions ? positions[j] : j; };
    auto held_for = [&](int j) {
        const int p = position(j);
        return p < a.first || (!all && p >= since);
    };
    int moves = 0;
    if (k > 0 && k < n) {
        const int run = (n + kSelect - 1) / kSelect, base = w * run * 64;   // this wave's places: base + 64 i + lane
        uint32_t key[kHeld];
        uint32_t flags = 0;   // bit i: kept for its position
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            const int j = base + 64 * i + lane;
            key[i] = 0;
            if (i < run && j < n) {
                key[i] = ordered(mass[j]);
                flags |= (uint32_t)held_for(j) << i;
            }
        }
        // f(place, its integer, whether it is kept for its position) for this lane's places, all lanes together
        auto each = [&](auto f) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < kHeld; ++i)
                if (i < run) {
                    const int j = base + 64 * i + lane;
                    f(j, j < n, key[i], (flags >> i & 1) != 0);
                }
            for (int i = kHeld; i < run; ++i) {
                const int j = base + 64 * i + lane;
                const bool in = j < n;
                f(j, in, in ? ordered(mass[j]) : 0u, in && held_for(j));
            }
        };
        // the sum of a wave's count over the workgroup; before: that of the waves before this one
        auto sum_waves = [&](uint32_t mine, uint32_t *room, uint32_t &before) {
            __syncthreads();
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
        };
        uint32_t mine = 0, before;
        each([&](int, bool in, uint32_t, bool held) { mine += __popcll(__ballot(in && held)); });
        const uint32_t kept = sum_waves(mine, wave_sum, before);
        // those that are kept for their positions all stay, and the rest comes from the others; or they are too many
        const bool of_held = kept > (uint32_t)k;
        uint32_t need = of_held ? k : k - kept;   // how many of the candidates stay
        uint32_t limit = 0, ties = 0, equal = 0;  // candidates over limit stay, and `ties` of the `equal` ones at it
        if (need > 0) {
            uint32_t mask = 0;
            for (int shift = 21; shift >= -1; shift -= 11) {   // bits 31-21, 20-10, 9-0
                const int at = max(shift, 0), width = shift < 0 ? 10 : 11;
                __syncthreads();
                for (int i = tid; i < kBins; i += kSelect) bins[i] = 0;
                __syncthreads();
                each([&](int, bool in, uint32_t x, bool held) {
                    if (in && held == of_held && (x & mask) == limit) atomicAdd(&bins[x >> at & ((1u << width) - 1)], 1u);
                });
                __syncthreads();
                // the highest bin with `need` candidates in it and those above; lane t has bins 2 t, 2 t + 1 from the top
                const uint32_t c0 = bins[kBins - 1 - 2 * tid], c1 = bins[kBins - 2 - 2 * tid];
                uint32_t incl = c0 + c1;
#pragma unroll
                for (int x = 1; x < 64; x *= 2) {
                    const uint32_t v = __shfl_up(incl, x);
                    if (lane >= x) incl += v;
                }
                const uint32_t total = __shfl(incl, 63);
                sum_waves(total, wave_sum, before);
                incl += before;
                const uint32_t below = incl - c0 - c1;
                if (below < need && need <= incl) {
                    const bool second = need > below + c0;
                    found_bin = kBins - 1 - 2 * tid - (second ? 1 : 0);
                    found_above = below + (second ? c0 : 0);
                    found_count = second ? c1 : c0;
                }
                __syncthreads();
                limit |= found_bin << at;
                mask |= ((1u << width) - 1) << at;
                need -= found_above;
                equal = found_count;
            }
            ties = need;
        }
        const bool any = ties > 0;   // some candidates stay
        uint32_t tie_rank = 0;   // of the next place of this wave at the limit
        if (ties < equal) {
            mine = 0;
            each([&](int, bool in, uint32_t x, bool held) { mine += __popcll(__ballot(in && held == of_held && x == limit)); });
            sum_waves(mine, wave_sum, tie_rank);
        }
        const unsigned long long lower = (1ull << lane) - 1;
        auto each_stay = [&](auto f) __attribute__((always_inline)) {
            uint32_t rank = tie_rank;
            each([&](int j, bool in, uint32_t x, bool held) {
                const bool candidate = in && held == of_held, tie = candidate && any && x == limit;
                const unsigned long long vote = __ballot(tie);
                const bool stays = in && (candidate ? any && (x > limit || (tie && rank + __popcll(vote & lower) < ties))
                                                    : held);
                rank += __popcll(vote);
                f(j, in, stays);
            });
        };
        uint32_t holes = 0, late = 0, hole_at, late_at;
        each_stay([&](int j, bool in, bool stays) {
            holes += __popcll(__ballot(in && !stays && j < k));
            late += __popcll(__ballot(stays && j >= k));
        });
        moves = (int)sum_waves(holes, wave_sum, hole_at);
        sum_waves(late, wave_two, late_at);
        int32_t *to = a.to + b * a.half, *from = a.from + b * a.half;
        each_stay([&](int j, bool in, bool stays) {
            const bool hole = in && !stays && j < k, moving = stays && j >= k;
            const unsigned long long h = __ballot(hole), m = __ballot(moving);
            if (hole) to[hole_at + __popcll(h & lower)] = j;
            if (moving) from[late_at + __popcll(m & lower)] = j;
            hole_at += __popcll(h);
            late_at += __popcll(m);
            if (stays && j < k) {
                if (moved_mass) mass_out[j] = mass[j];
                if (moved_positions) positions_out[j] = position(j);
            }
        });
        __syncthreads();
        for (int i = tid; i < moves; i += kSelect) {
            mass_out[to[i]] = mass[from[i]];
            positions_out[to[i]] = position(from[i]);
        }
    } else {
        for (int j = tid; j < k; j += kSelect) {
            if (moved_mass) mass_out[j] = mass[j];
            if (moved_positions) positions_out[j] = position(j);
        }
    }
    __syncthreads();   // what moves, and the length, which may be written where it was, has been read
    if (tid == 0) {
        a.lens_out[b] = k;
        a.counts[b] = moves;
    }
    for (int j = k + tid; j < a.capacity; j += kSelect) {
        mass_out[j] = 0.0f;
        positions_out[j] = -1;
    }
}

__global__ __launch_bounds__(kThreads) void move_kernel(EvictArgs a) {
    constexpr int AHEAD = 4;   // moves on their way
    const int b = (int)(blockIdx.x / (unsigned)a.shares), share = (int)(blockIdx.x % (unsigned)a.shares);
    const int moves = a.counts[b];
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
            uint4 v[AHEAD];
#pragma unroll
            for (int q = 0; q < AHEAD; ++q)
                if (i + q * (long long)step < moves) v[q] = *reinterpret_cast<const uint4 *>(row(from[i + q * step]));
#pragma unroll
            for (int q = 0; q < AHEAD; ++q)
                if (i + q * (long long)step < moves) *reinterpret_cast<uint4 *>(row(to[i + q * step])) = v[q];
        }
    }
}

}  // namespace

hipError_t launch_evict(const EvictArgs &a, hipStream_t st) {
    select_kernel<<<(unsigned)a.batch, kSelect, 0, st>>>(a);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    move_kernel<<<(unsigned)a.batch * a.shares, kThreads, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace ftcnn
