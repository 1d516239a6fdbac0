// The C entry points of what differs from request to request (include/ftcnn.h): adapters, attention weights and eviction.
// Argument checks and the launch plans.
#include <math.h>

#include <algorithm>

#include "evict.h"
#include "low_rank.h"
#include "mass.h"

namespace ftcnn {
namespace {

#define FT_REQUESTS_HIP(expr, where)                                                     \
    do {                                                                                 \
        const hipError_t _e = (expr);                                                    \
        if (_e != hipSuccess) return set_error(FTCNN_E_HIP, "%s: %s", where, hipGetErrorString(_e)); \
    } while (0)

constexpr long long kMaxRows = 1LL << 30;   // as in paged_api.hip
constexpr float kLog2E = 1.44269504088896340736f;
constexpr long long kMaxThreads = (1LL << 32) - 1;   // of a launch
constexpr int kMaxRank = 128;

template <typename... P> bool aligned16(P... p) { return ((reinterpret_cast<uintptr_t>(p) % 16 == 0) && ...); }
template <typename... S> bool whole_units(int vec, S... s) { return ((s % vec == 0) && ...); }
int vec_of(int32_t dtype) { return dtype == FTCNN_F32 ? 4 : 8; }
size_t up256(size_t x) { return (x + 255) & ~size_t(255); }

int check_dtype(int32_t dtype, const char *what) {
    if (dtype != FTCNN_F32 && dtype != FTCNN_BF16) return set_error(FTCNN_E_DTYPE, "%s: dtype %d", what, dtype);
    return FTCNN_OK;
}
int check_workspace(const char *what, size_t bytes, const void *workspace) {
    if (bytes && (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256))
        return set_error(FTCNN_E_WORKSPACE, "%s: workspace missing or not 256-byte aligned", what);
    return FTCNN_OK;
}
// The cache of a call: sizes of it and of the page lists.
int check_cache(const char *what, int32_t batch, int32_t kv_heads, int32_t dim, int32_t pages, int32_t page, int32_t list_len) {
    if (batch < 0 || kv_heads < 1 || pages < 1 || page < 1 || list_len < 0)
        return set_error(FTCNN_E_SHAPE, "%s: non-positive size", what);
    if (dim < 8 || dim > 256 || dim % 8)
        return set_error(FTCNN_E_UNSUPPORTED, "%s: dim %d (a multiple of 8, at most 256)", what, dim);
    if ((long long)list_len * page > kMaxRows) return set_error(FTCNN_E_SHAPE, "%s: more than 2^30 rows", what);
    if ((long long)batch * kv_heads > kMaxRows)
        return set_error(FTCNN_E_SHAPE, "%s: %d sequences of %d key heads", what, batch, kv_heads);
    return FTCNN_OK;
}
int check_cache_strides(const char *what, int vec, const int64_t *stride) {
    for (int i = 0; i < 3; ++i)
        if (stride[i] < 0 || stride[i] > kMaxRows / 2)
            return set_error(FTCNN_E_UNSUPPORTED, "%s: cache strides are 0 to 2^29 elements", what);
    if (!whole_units(vec, stride[0], stride[1], stride[2]))
        return set_error(FTCNN_E_UNSUPPORTED, "%s: rows of the cache must start on 16 bytes", what);
    return FTCNN_OK;
}
// Rows of one value a place: those of two sequences must not share any that is written.
int check_places(const char *what, const char *name, int32_t batch, long long capacity, int64_t stride) {
    if (batch > 1 && stride < capacity)
        return set_error(FTCNN_E_UNSUPPORTED, "%s: %s of a sequence every %lld, for %lld places", what, name,
                         (long long)stride, capacity);
    return FTCNN_OK;
}

int check_low_rank(const ftcnn_low_rank_desc *d) {
    const char *what = "low_rank_add";
    if (!d) return set_error(FTCNN_E_ARG, "%s: null descriptor", what);
    const int rc = check_dtype(d->dtype, what);
    if (rc != FTCNN_OK) return rc;
    if (d->tokens < 0 || d->ch < 1 || d->m < 1 || d->adapters < 1 || d->rank < 1)
        return set_error(FTCNN_E_SHAPE, "%s: non-positive size", what);
    const int vec = vec_of(d->dtype);
    if (!whole_units(vec, d->ch, d->m, d->rank) || d->rank > kMaxRank)
        return set_error(FTCNN_E_UNSUPPORTED, "%s: ch %d, m %d, rank %d (multiples of %d, the rank at most %d)", what, d->ch,
                         d->m, d->rank, vec, kMaxRank);
    if (!whole_units(vec, d->x_stride, d->y_stride, d->out_stride, d->a_stride[0], d->a_stride[1], d->b_stride[0],
                     d->b_stride[1]))
        return set_error(FTCNN_E_UNSUPPORTED, "%s: rows of tokens and adapters must start on 16 bytes", what);
    if (d->tokens > kMaxRows || d->ch > kMaxRows || d->m > kMaxRows)
        return set_error(FTCNN_E_SHAPE, "%s: more than 2^30 tokens, channels or outputs", what);
    if (d->tokens) {
        const LowRankPlan p = low_rank_plan(*d);
        // (of 512 threads: the first launch, unless tokens are grouped, and the one for both products)
        const long long one = p.both ? 0 : (long long)p.tiles * p.ways * p.splits * p.groups;
        const long long two = (long long)((p.tiles + p.together - 1) / p.together) * p.expand_ways * p.spans;
        if (std::max((p.grouped ? 1 : 2) * one, (p.both ? 2 : 1) * two) > kMaxThreads / kThreads)
            return set_error(FTCNN_E_SHAPE, "%s: %lld and %lld workgroups", what, one, two);
    }
    return FTCNN_OK;
}

int check_mass(const ftcnn_mass_desc *d) {
    const char *what = "attention_mass";
    if (!d) return set_error(FTCNN_E_ARG, "%s: null descriptor", what);
    int rc = check_dtype(d->dtype, what);
    if (rc != FTCNN_OK) return rc;
    if (d->tokens < 0 || d->heads < 1 || d->max_q < 0 || d->max_kv < 0)
        return set_error(FTCNN_E_SHAPE, "%s: non-positive size", what);
    rc = check_cache(what, d->batch, d->kv_heads, d->dim, d->pages, d->page, d->list_len);
    if (rc != FTCNN_OK) return rc;
    if (d->heads % d->kv_heads)
        return set_error(FTCNN_E_SHAPE, "%s: %d key heads do not divide %d heads", what, d->kv_heads, d->heads);
    if ((long long)d->tokens * d->heads > kMaxRows) return set_error(FTCNN_E_SHAPE, "%s: more than 2^30 rows", what);
    if (d->window < 0 || (d->window > 0 && !d->causal))
        return set_error(FTCNN_E_ARG, "%s: window %d (0, or positive with causal)", what, d->window);
    if (!(d->scale > 0.0f) || !std::isfinite(d->scale * kLog2E))
        return set_error(FTCNN_E_ARG, "%s: scale %g (positive, below 2.3e38)", what, (double)d->scale);
    return FTCNN_OK;
}

int check_evict(const ftcnn_evict_desc *d) {
    const char *what = "evict";
    if (!d) return set_error(FTCNN_E_ARG, "%s: null descriptor", what);
    int rc = check_dtype(d->dtype, what);
    if (rc != FTCNN_OK) return rc;
    if (d->max_kv < 0) return set_error(FTCNN_E_SHAPE, "%s: max_kv %d", what, d->max_kv);
    if (d->first < 0) return set_error(FTCNN_E_ARG, "%s: first %d", what, d->first);
    rc = check_cache(what, d->batch, d->kv_heads, d->dim, d->pages, d->page, d->list_len);
    if (rc != FTCNN_OK) return rc;
    if ((long long)d->batch * 1024 > kMaxThreads) return set_error(FTCNN_E_SHAPE, "%s: %d sequences", what, d->batch);
    if ((long long)d->kv_heads * (d->dim / vec_of(d->dtype)) > kMaxRows / 2)   // move_kernel counts those of keys and values
        return set_error(FTCNN_E_SHAPE, "%s: %d key heads of %d", what, d->kv_heads, d->dim);
    return FTCNN_OK;
}

struct EvictRoom {
    size_t from, to, part, bytes;   // after the moves' counts
    long long half;                 // moves of a sequence, at most
    int parts;
};
long long evict_longest(const ftcnn_evict_desc &d) {
    const long long capacity = (long long)d.list_len * d.page;
    return std::min(d.max_kv > 0 ? d.max_kv : capacity, capacity);
}
EvictRoom evict_room(const ftcnn_evict_desc &d) {
    EvictRoom r{};
    if (d.batch == 0) return r;
    const long long capacity = (long long)d.list_len * d.page;
    r.half = std::max(1LL, capacity / 2);
    const size_t list = up256((size_t)d.batch * r.half * sizeof(int32_t));
    r.from = up256((size_t)d.batch * sizeof(int32_t));
    r.to = r.from + list;
    r.part = r.to + list;
    const long long parts = (capacity + kEvictPart - 1) / kEvictPart;
    // (16384 rows 26 us with a workgroup for the sequence, 16400 in parts 32; 131072 in parts 36, with one workgroup 367)
    if (evict_longest(d) > kEvictHeld && d.batch * parts * 1024 <= kMaxThreads) r.parts = (int)parts;
    r.bytes = r.part + (size_t)d.batch * r.parts * sizeof(EvictPart);
    return r;
}

}  // namespace

MassPlan mass_plan(const ftcnn_mass_desc &d) {
    MassPlan p{};
    const long long capacity = (long long)d.list_len * d.page;
    if (d.batch == 0 || d.tokens == 0 || capacity == 0) return p;
    const long long group = d.heads / d.kv_heads;
    const long long max_q = std::max(1LL, std::min<long long>(d.max_q > 0 ? d.max_q : d.tokens, d.tokens));
    const long long max_kv = std::max(1LL, std::min(d.max_kv > 0 ? d.max_kv : capacity, capacity));
    const long long rows = max_q * group;
    const int es = d.dtype == FTCNN_F32 ? 4 : 2;
    p.dp = d.dim <= 64 ? 64 : (d.dim <= 128 ? 128 : 256);
    p.wide = rows > 64;
    const bool narrow = p.dp * es <= 256;
    p.head_parts = p.row_parts = 1;
    p.keys = narrow ? 32 : 16;
    if (p.wide) {
        // Parts of at most 2^28 bytes.  A key head is a workgroup's, and its rows are shared by so many that there are two
        // workgroups to a compute unit, of two tiles of 64 rows at least, or eight, so that long ones even out, of eight
        // tiles (two prompts of 8192 tokens 560 us, four 602; 512 tokens over 8704 keys, which have 32 tiles, 61 with four
        // workgroups to a compute unit, 73 with eight).  Parts are rounded up: workgroups that are a few more than the device holds
        // at a time take another round (129 tokens over 22677 keys, one key head: 540, of which 512 at a time).
        const long long room = (1LL << 26) / (d.batch * capacity), tiles = (rows + 63) / 64;
        auto split = [&](int keys) {
            p.keys = keys;
            p.head_parts = (int)std::max(1LL, std::min<long long>(d.kv_heads, room));
            const long long base = (max_kv + keys - 1) / keys * d.batch * p.head_parts;
            auto share = [&](long long want, long long least) { return std::min(tiles / least, (want * kComputeUnits + base - 1) / base); };
            p.row_parts = (int)std::max(1LL, std::min(std::max(share(2, 2), share(8, 8)), room / p.head_parts));
            return base * p.row_parts;
        };
        // a wave has 64 keys where registers hold them (those prompts 582 us; 32 650), 32 where there are too few
        // workgroups otherwise (3 x 257 tokens over 1257 keys, fp32, heads of 64: 27 us; 64 keys 37)
        if (!narrow || split(256) < 2 * kComputeUnits) split(128);
        if (p.head_parts * p.row_parts > 1)
            p.bytes = up256((size_t)p.head_parts * p.row_parts * d.batch * capacity * sizeof(float));
    }
    const long long blocks = (max_kv + p.keys - 1) / p.keys;
    if (!p.wide) {   // as many workgroups as are on the device at a time
        p.blocks = (int)std::min(blocks * d.batch, (long long)kComputeUnits * (narrow ? 3 : 2));
        return p;
    }
    // a workgroup goes on to block b + p.blocks
    const long long most = kMaxThreads / kThreads / ((long long)d.batch * p.head_parts * p.row_parts);
    p.blocks = (int)std::max(1LL, std::min(blocks, most));
    return p;
}

}  // namespace ftcnn

using namespace ftcnn;

extern "C" {

size_t ftcnn_low_rank_workspace_bytes(const ftcnn_low_rank_desc *desc) {
    return check_low_rank(desc) == FTCNN_OK ? low_rank_plan(*desc).bytes : 0;
}

int ftcnn_low_rank_add(const ftcnn_low_rank_desc *d, const void *y, const void *x, const void *a, const void *b,
                       const int32_t *ids, const float *scales, const int32_t *ranks, void *out, void *workspace,
                       hipStream_t stream) {
    const char *what = "low_rank_add";
    int rc = check_low_rank(d);
    if (rc != FTCNN_OK) return rc;
    if (d->tokens == 0) return FTCNN_OK;
    if (!y || !x || !a || !b || !ids || !out) return set_error(FTCNN_E_ARG, "%s: null pointer", what);
    if (!aligned16(y, x, a, b, out))
        return set_error(FTCNN_E_UNSUPPORTED, "%s: rows of tokens and adapters must start on 16 bytes", what);
    if (out == y && d->tokens > 1 && d->out_stride != d->y_stride)
        return set_error(FTCNN_E_ARG, "%s: out is y with other strides", what);
    if (d->tokens > 1 && d->out_stride < d->m)
        return set_error(FTCNN_E_UNSUPPORTED, "%s: out's tokens overlap", what);
    const LowRankPlan pl = low_rank_plan(*d);
    rc = check_workspace(what, pl.bytes, workspace);
    if (rc != FTCNN_OK) return rc;
    LowRankArgs g{};
    g.x = x;
    g.y = y;
    g.a = a;
    g.b = b;
    g.out = out;
    g.scales = scales;
    g.ranks = ranks;
    g.ids = ids;
    char *ws = static_cast<char *>(workspace);
    g.low = static_cast<float *>(workspace);
    if (pl.grouped) {
        g.records = reinterpret_cast<int4 *>(ws + pl.records);
        g.grouped = reinterpret_cast<int32_t *>(ws + pl.order);
        g.counts = reinterpret_cast<int32_t *>(ws + pl.count);
        g.slots = pl.slots;
        g.div_slots = fast_div((uint32_t)pl.slots);
    }
    g.xs = d->x_stride;
    g.ys = d->y_stride;
    g.os = d->out_stride;
    for (int i = 0; i < 2; ++i) {
        g.as[i] = d->a_stride[i];
        g.bs[i] = d->b_stride[i];
    }
    g.tokens = d->tokens;
    g.ch = d->ch;
    g.m = d->m;
    g.adapters = d->adapters;
    g.rank = d->rank;
    g.groups = pl.groups;
    g.splits = pl.splits;
    g.div_splits = fast_div((uint32_t)pl.splits);
    g.ways = pl.ways;
    g.expand_ways = pl.expand_ways;
    g.columns = pl.columns;
    g.div_groups = fast_div((uint32_t)pl.groups);
    g.div_ways = fast_div((uint32_t)pl.ways);
    g.div_expand_ways = fast_div((uint32_t)pl.expand_ways);
    g.div_spans = fast_div((uint32_t)pl.spans);
    FT_REQUESTS_HIP(launch_low_rank(d->dtype, pl, g, stream), what);
    return FTCNN_OK;
}

size_t ftcnn_attention_mass_workspace_bytes(const ftcnn_mass_desc *desc) {
    return check_mass(desc) == FTCNN_OK ? mass_plan(*desc).bytes : 0;
}

int ftcnn_attention_mass(const ftcnn_mass_desc *d, const void *q, const void *k_cache, const int32_t *page_list,
                         const int32_t *kv_lens, const int32_t *q_starts, const float *lse, float *mass, void *workspace,
                         hipStream_t stream) {
    const char *what = "attention_mass";
    int rc = check_mass(d);
    if (rc != FTCNN_OK) return rc;
    if (!q_starts && d->tokens != d->batch)
        return set_error(FTCNN_E_SHAPE, "%s: %d tokens of %d sequences need q_starts", what, d->tokens, d->batch);
    const long long capacity = (long long)d->list_len * d->page;
    if (d->tokens == 0 || d->batch == 0 || capacity == 0) return FTCNN_OK;
    if (!q || !k_cache || !page_list || !kv_lens || !lse || !mass) return set_error(FTCNN_E_ARG, "%s: null pointer", what);
    const int vec = vec_of(d->dtype);
    rc = check_cache_strides(what, vec, d->k_cache_stride);
    if (rc == FTCNN_OK) rc = check_places(what, "mass", d->batch, capacity, d->mass_stride);
    if (rc != FTCNN_OK) return rc;
    if (!aligned16(q, k_cache) || !whole_units(vec, d->q_stride[0], d->q_stride[1]))
        return set_error(FTCNN_E_UNSUPPORTED, "%s: rows of q and the cache must start on 16 bytes", what);
    const MassPlan pl = mass_plan(*d);
    rc = check_workspace(what, pl.bytes, workspace);
    if (rc != FTCNN_OK) return rc;
    const long long blocks = pl.wide ? (long long)pl.blocks * d->batch * pl.head_parts * pl.row_parts : pl.blocks;
    if (blocks > kMaxThreads / kThreads) return set_error(FTCNN_E_SHAPE, "%s: %lld workgroups", what, blocks);
    MassArgs m{};
    AttnArgs &t = m.t;
    t.q = q;
    t.k = k_cache;
    t.page_list = page_list;
    t.kv_lens = kv_lens;
    t.q_starts = q_starts;
    for (int i = 0; i < 3; ++i) {
        if (i < 2) t.qs[i] = d->q_stride[i];
        t.kb[i] = (unsigned)(d->k_cache_stride[i] * (16 / vec));
    }
    t.list_stride = d->list_stride;
    t.batch = d->batch;
    t.tokens = d->tokens;
    t.kv_heads = d->kv_heads;
    t.group = d->heads / d->kv_heads;
    t.dim = d->dim;
    t.pages = d->pages;
    t.page = d->page;
    t.capacity = (int)capacity;
    t.causal = d->causal != 0;
    t.window = (int)std::min<long long>(d->window, capacity);   // a wider one hides nothing more
    t.div_page = fast_div((uint32_t)d->page);
    t.div_group = fast_div((uint32_t)t.group);
    t.scale_log2 = d->scale * kLog2E;
    m.lse = lse;
    m.mass = mass;
    m.part = static_cast<float *>(workspace);
    m.mass_stride = d->mass_stride;
    m.blocks = pl.blocks;
    m.head_parts = pl.head_parts;
    m.row_parts = pl.row_parts;
    m.div_heads = fast_div((uint32_t)pl.head_parts);
    m.div_rows = fast_div((uint32_t)pl.row_parts);
    m.div_blocks = fast_div((uint32_t)pl.blocks);
    m.near = d->q_stride[0] >= 0 && d->q_stride[0] < 1 << 24 && d->q_stride[1] >= 0 && d->q_stride[1] < 1 << 23;
    FT_REQUESTS_HIP(d->dtype == FTCNN_F32 ? launch_mass_f32(pl, m, stream) : launch_mass_bf16(pl, m, stream), what);
    if (pl.bytes) FT_REQUESTS_HIP(launch_mass_join(pl, m, stream), "attention_mass: join");
    return FTCNN_OK;
}

size_t ftcnn_evict_workspace_bytes(const ftcnn_evict_desc *desc) {
    return check_evict(desc) == FTCNN_OK ? evict_room(*desc).bytes : 0;
}

int ftcnn_evict(const ftcnn_evict_desc *d, void *k_cache, void *v_cache, const int32_t *page_list, const int32_t *kv_lens,
                const int32_t *keep, const float *mass, const int32_t *positions, const int32_t *since, int32_t *lens_out,
                float *mass_out, int32_t *positions_out, void *workspace, hipStream_t stream) {
    const char *what = "evict";
    int rc = check_evict(d);
    if (rc != FTCNN_OK) return rc;
    if (d->batch == 0) return FTCNN_OK;
    const long long capacity = (long long)d->list_len * d->page;
    if (!kv_lens || !keep || !lens_out ||
        (capacity && (!k_cache || !v_cache || !page_list || !mass || !mass_out || !positions_out)))
        return set_error(FTCNN_E_ARG, "%s: null pointer", what);
    const int vec = vec_of(d->dtype);
    rc = check_cache_strides(what, vec, d->k_cache_stride);
    if (rc == FTCNN_OK) rc = check_cache_strides(what, vec, d->v_cache_stride);
    if (rc == FTCNN_OK) rc = check_places(what, "mass_out", d->batch, capacity, d->mass_out_stride);
    if (rc == FTCNN_OK) rc = check_places(what, "positions_out", d->batch, capacity, d->position_out_stride);
    if (rc != FTCNN_OK) return rc;
    if (mass == mass_out && d->batch > 1 && d->mass_stride != d->mass_out_stride)
        return set_error(FTCNN_E_ARG, "%s: mass_out is mass with other strides", what);
    if (positions == positions_out && d->batch > 1 && d->position_stride != d->position_out_stride)
        return set_error(FTCNN_E_ARG, "%s: positions_out is positions with other strides", what);
    if (!aligned16(k_cache, v_cache))
        return set_error(FTCNN_E_UNSUPPORTED, "%s: rows of the cache must start on 16 bytes", what);
    const EvictRoom room = evict_room(*d);
    rc = check_workspace(what, room.bytes, workspace);
    if (rc != FTCNN_OK) return rc;
    EvictArgs e{};
    e.k = k_cache;
    e.v = v_cache;
    for (int i = 0; i < 3; ++i) {
        e.kb[i] = (unsigned)(d->k_cache_stride[i] * (16 / vec));
        e.vb[i] = (unsigned)(d->v_cache_stride[i] * (16 / vec));
    }
    e.page_list = page_list;
    e.kv_lens = kv_lens;
    e.keep = keep;
    e.positions = positions;
    e.since = since;
    e.mass = mass;
    e.lens_out = lens_out;
    e.mass_out = mass_out;
    e.positions_out = positions_out;
    e.list_stride = d->list_stride;
    e.ms = d->mass_stride;
    e.ps = d->position_stride;
    e.mos = d->mass_out_stride;
    e.pos = d->position_out_stride;
    e.batch = d->batch;
    e.kv_heads = d->kv_heads;
    e.pages = d->pages;
    e.page = d->page;
    e.capacity = (int)capacity;
    e.first = d->first;
    e.units = d->dim / vec;
    char *ws = static_cast<char *>(workspace);
    e.counts = reinterpret_cast<int32_t *>(ws);
    e.from = reinterpret_cast<int32_t *>(ws + room.from);
    e.to = reinterpret_cast<int32_t *>(ws + room.to);
    e.half = room.half;
    e.parts = room.parts;
    e.part = reinterpret_cast<EvictPart *>(ws + room.part);
    e.div_page = fast_div((uint32_t)d->page);
    // workgroups of a sequence: four rows of its moves each at a time, 2048 in all (64 sequences of 32768 rows of 256 bytes
    // halved 123 us, 132 with 1024; those that find nothing to move cost a microsecond)
    const long long longest = evict_longest(*d);
    e.held = (int)std::min<long long>(room.parts ? kEvictPart : kEvictHeld, std::max(1024LL, (longest + 1023) / 1024 * 1024));
    const long long together = std::max(1LL, (long long)kThreads / (2LL * d->kv_heads * e.units));
    e.shares = (int)std::max(1LL, std::min((longest / 2 + 4 * together - 1) / (4 * together), 2048LL / d->batch));
    FT_REQUESTS_HIP(launch_evict(e, stream), what);
    return FTCNN_OK;
}

}  // extern "C"
