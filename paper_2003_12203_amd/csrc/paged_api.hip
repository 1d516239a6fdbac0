// The C entry points of the serving operators (include/ftcnn.h): argument checks and the launch plan.
#include <math.h>

#include <algorithm>

#include "paged.h"

namespace ftcnn {
namespace {

#define FT_PAGED_HIP(expr, where)                                                        \
    do {                                                                                 \
        const hipError_t _e = (expr);                                                    \
        if (_e != hipSuccess) return set_error(FTCNN_E_HIP, "%s: %s", where, hipGetErrorString(_e)); \
    } while (0)

// Rows a sequence's page list can name, rows of queries, key heads of all sequences.  attn_plan's products of units
// and keys then stay below 2^63.
constexpr long long kMaxRows = 1LL << 30;
constexpr float kLog2E = 1.44269504088896340736f;
constexpr long long kMaxThreads = (1LL << 32) - 1;   // of a launch

bool aligned16(const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

int check_dtype(int32_t dtype, const char *what) {
    if (dtype != FTCNN_F32 && dtype != FTCNN_BF16) return set_error(FTCNN_E_DTYPE, "%s: dtype %d", what, dtype);
    return FTCNN_OK;
}

// What the two rotating operators share: sizes, the rotation, the weights.
int check_rope(const char *what, int32_t dtype, int32_t tokens, int32_t heads, int32_t dim, int32_t rot,
               int32_t layout, int32_t max_pos, float eps, const void *positions, const void *table,
               bool normed, int32_t weight_dtype) {
    const int rc = check_dtype(dtype, what);
    if (rc != FTCNN_OK) return rc;
    if (tokens < 0 || heads < 1 || dim < 2 || dim > 256 || dim % 2)
        return set_error(FTCNN_E_SHAPE, "%s: tokens %d, heads %d, dim %d (even, at most 256)", what, tokens, heads,
                         dim);
    if ((long long)tokens * heads > kMaxRows) return set_error(FTCNN_E_SHAPE, "%s: more than 2^30 rows", what);
    if (!positions != !table) return set_error(FTCNN_E_ARG, "%s: positions and table go together", what);
    if (positions) {
        if (rot < 2 || rot % 2 || rot > dim)
            return set_error(FTCNN_E_SHAPE, "%s: rot %d (even, 2 to dim = %d)", what, rot, dim);
        if (max_pos < 1) return set_error(FTCNN_E_SHAPE, "%s: max_pos %d", what, max_pos);
        if (layout != FTCNN_ROPE_HALF && layout != FTCNN_ROPE_INTERLEAVED)
            return set_error(FTCNN_E_ARG, "%s: layout %d", what, layout);
    }
    if (normed) {
        if (!(eps >= 0.0f) || !std::isfinite(eps)) return set_error(FTCNN_E_ARG, "%s: eps %g", what, (double)eps);
        if (weight_dtype != FTCNN_F32 && weight_dtype != dtype)
            return set_error(FTCNN_E_DTYPE, "%s: weights of dtype %d (fp32, or the tensors')", what, weight_dtype);
    }
    return FTCNN_OK;
}

}  // namespace

static int attn_threads(const AttnPlan &p) { return p.rows == 16 ? 64 : 256; }   // of a workgroup

AttnPlan attn_plan(const ftcnn_attention_desc &d) {
    AttnPlan p{};
    if (d.batch == 0 || d.tokens == 0) return p;   // no units
    const long long group = d.heads / d.kv_heads, capacity = (long long)d.list_len * d.page;
    const long long max_q = std::max(1LL, std::min<long long>(d.max_q > 0 ? d.max_q : d.tokens, d.tokens));
    const long long max_kv = std::max(1LL, std::min(d.max_kv > 0 ? d.max_kv : capacity, capacity));
    const long long rows = max_q * group;
    p.dp = d.dim <= 64 ? 64 : (d.dim <= 128 ? 128 : 256);
    const bool bf = d.dtype == FTCNN_BF16;
    const long long es = bf ? 2 : 4;
    // up to 16 rows a wave alone; more, a workgroup of four waves (32 rows of 30000 keys: 46 us, two tiles of 16
    // of them in one wave 96; 64 rows: 64 us, a workgroup of two waves 143)
    const bool wide = rows > 16;
    p.rows = wide ? 128 : 16;
    p.keys = wide ? (bf && p.dp <= 128 ? 64 : 32) : (p.dp * es <= 256 ? 32 : 16);
    const long long tile = p.rows;
    const long long tiles = (rows + tile - 1) / tile;
    // A workgroup goes on to tile t + p.tiles, so fewer do as well where all of them (without a hint of the longest
    // sequence most have nothing to do) would pass what a launch holds.
    const long long most = kMaxThreads / attn_threads(p) / ((long long)d.batch * d.kv_heads);
    p.tiles = (int)std::min(tiles, std::max(1LL, most));
    // workgroups that are on the device at a time (registers and LDS)
    const bool narrow = p.dp * es <= 256;
    const long long fit = kComputeUnits * (wide ? (p.dp <= 128 ? 2 : 1) : (narrow ? 8 : 4));
    const long long some = std::min<long long>((long long)d.batch * tiles, d.tokens * group / tile + d.batch);
    const long long units = some * d.kv_heads;
    const long long range = d.window > 0 ? std::min<long long>(max_kv, d.window + tile / group + 1) : max_kv;
    // Whole units or even runs: the shorter by the sizes the host knows, in the time of a key (a wave alone
    // 70 ns; a workgroup, bf16 25 ns, fp32 60 ns).  What the start and end of a unit take: a wave one tile, bf16
    // workgroups five of 64 keys (mixed chunks 117 us; three 130, one 153), fp32 two of 32.  What even runs
    // take besides, the schedule and the join: 14 us of a wave, 25 of a workgroup.  A run is not made shorter than
    // min_run.  All of it was measured with heads of 64 and 128, and is applied to others as it is.  Whole / even: one
    // prompt of 512 tokens 18 / 44 us, of 2048 56 / 88; chunks over 8192 cached tokens 256 / 111; 64 tokens over
    // 500 keys 44 / 44, over 2000 169 / 114.
    p.min_run = wide ? 128 : 64;
    p.unit_cost = wide ? (bf ? 320 : 64) : 32;
    const long long rest = wide ? (bf ? 1100 : 330) : 200;
    const long long mean = d.window > 0 || !d.causal ? range : std::max(1LL, max_kv - max_q / 2);
    const long long whole = std::max(range, units * mean / fit) + p.unit_cost * ((units + fit - 1) / fit);
    // as many runs on every compute unit: 365 on 256 of them 53 us, 256 runs 42; fp32 workgroups, whose matrix
    // instructions leave a second one nothing, one each: 200 tokens over 6000, heads of 128, 125 us, two 138
    long long runs = std::min(wide && !bf ? kComputeUnits : fit, (units * range + p.min_run - 1) / p.min_run);
    if (runs > kComputeUnits) runs -= runs % kComputeUnits;
    const long long even = units * (mean + p.unit_cost) / runs + rest;
    if (even < whole) {
        p.groups = (int)runs;
        p.part_rows = (int)std::min<long long>(tile, d.tokens * group);
        p.join_rows = wide ? 8 : (p.groups >= 32 * units ? 1 : 16);
        const size_t n = 2 * (size_t)p.groups * p.part_rows;
        auto up = [](size_t x) { return (x + 255) & ~size_t(255); };
        p.part_ml = up(n * d.dim * sizeof(float));
        p.cuts = p.part_ml + up(n * 2 * sizeof(float));
        p.bytes = p.cuts + up(p.groups * sizeof(AttnCut));
    }
    return p;
}

namespace {

int check_attention(const ftcnn_attention_desc *d) {
    const char *what = "paged_attention";
    if (!d) return set_error(FTCNN_E_ARG, "%s: null descriptor", what);
    const int rc = check_dtype(d->dtype, what);
    if (rc != FTCNN_OK) return rc;
    if (d->batch < 0 || d->tokens < 0 || d->heads < 1 || d->kv_heads < 1 || d->pages < 1 || d->page < 1 ||
        d->list_len < 0 || d->max_q < 0 || d->max_kv < 0)
        return set_error(FTCNN_E_SHAPE, "%s: non-positive size", what);
    if (d->heads % d->kv_heads)
        return set_error(FTCNN_E_SHAPE, "%s: %d key heads do not divide %d heads", what, d->kv_heads, d->heads);
    if (d->dim < 8 || d->dim > 256 || d->dim % 8)
        return set_error(FTCNN_E_UNSUPPORTED, "%s: dim %d (a multiple of 8, at most 256)", what, d->dim);
    if ((long long)d->tokens * d->heads > kMaxRows || (long long)d->list_len * d->page > kMaxRows)
        return set_error(FTCNN_E_SHAPE, "%s: more than 2^30 rows", what);
    if ((long long)d->batch * d->kv_heads > kMaxRows)
        return set_error(FTCNN_E_SHAPE, "%s: %d sequences of %d key heads", what, d->batch, d->kv_heads);
    if (d->window < 0 || (d->window > 0 && !d->causal))
        return set_error(FTCNN_E_ARG, "%s: window %d (0, or positive with causal)", what, d->window);
    if (!(d->scale > 0.0f) || !std::isfinite(d->scale * kLog2E))   // (the kernels take that product)
        return set_error(FTCNN_E_ARG, "%s: scale %g (positive, below 2.3e38)", what, (double)d->scale);
    return FTCNN_OK;
}

}  // namespace
}  // namespace ftcnn

using namespace ftcnn;

extern "C" {

int ftcnn_rope_table(const ftcnn_rope_scaling *sc, float *table, hipStream_t stream) {
    if (!sc || !table) return set_error(FTCNN_E_ARG, "rope_table: null pointer");
    if (sc->max_pos < 1 || sc->rot < 2 || sc->rot % 2 || sc->rot > 256)
        return set_error(FTCNN_E_SHAPE, "rope_table: max_pos %d, rot %d (even, at most 256)", sc->max_pos, sc->rot);
    if (sc->scaling < FTCNN_ROPE_PLAIN || sc->scaling > FTCNN_ROPE_PARTS)
        return set_error(FTCNN_E_ARG, "rope_table: scaling %d", sc->scaling);
    if (!(sc->base > 0.0) || !std::isfinite(sc->base) || !std::isfinite(sc->amplitude))
        return set_error(FTCNN_E_ARG, "rope_table: base %g, amplitude %g", sc->base, sc->amplitude);
    if (sc->scaling != FTCNN_ROPE_PLAIN && (!(sc->factor > 0.0) || !std::isfinite(sc->factor)))
        return set_error(FTCNN_E_ARG, "rope_table: factor %g", sc->factor);
    if (sc->scaling == FTCNN_ROPE_PARTS && (sc->original < 1 || !(sc->high > sc->low) || !std::isfinite(sc->low) ||
                                            !std::isfinite(sc->high)))
        return set_error(FTCNN_E_ARG, "rope_table: original %d, low %g, high %g", sc->original, sc->low, sc->high);
    FT_PAGED_HIP(launch_rope_table(*sc, table, stream), "rope_table");
    return FTCNN_OK;
}

int ftcnn_qk_norm_rope(const ftcnn_rope_desc *d, const void *q, const void *k, const int32_t *positions,
                       const float *table, const void *q_weight, const void *k_weight, void *q_out, void *k_out,
                       hipStream_t stream) {
    const char *what = "qk_norm_rope";
    if (!d) return set_error(FTCNN_E_ARG, "%s: null descriptor", what);
    if (d->heads < 0 || d->kv_heads < 0 || (long long)d->heads + d->kv_heads > kMaxRows)
        return set_error(FTCNN_E_SHAPE, "%s: heads %d and %d", what, d->heads, d->kv_heads);
    const int rc = check_rope(what, d->dtype, d->tokens, d->heads + d->kv_heads, d->dim, d->rot, d->layout,
                              d->max_pos, d->eps, positions, table, q_weight || k_weight, d->weight_dtype);
    if (rc != FTCNN_OK) return rc;
    if (d->tokens == 0) return FTCNN_OK;
    if ((d->heads && (!q || !q_out)) || (d->kv_heads && (!k || !k_out)))
        return set_error(FTCNN_E_ARG, "%s: null pointer", what);
    RopeArgs a{};
    const void *in[2] = {q, k}, *wt[2] = {q_weight, k_weight};
    void *out[2] = {q_out, k_out};
    const int32_t heads[2] = {d->heads, d->kv_heads};
    const int64_t *is[2] = {d->q_stride, d->k_stride}, *os[2] = {d->q_out_stride, d->k_out_stride};
    for (int s = 0; s < 2; ++s) {
        a.x[s] = in[s];
        a.y[s] = out[s];
        a.weight[s] = wt[s];
        a.heads[s] = heads[s];
        for (int i = 0; i < 2; ++i) {
            a.xs[s][i] = is[s][i];
            a.ys[s][i] = os[s][i];
        }
    }
    a.tokens = d->tokens;
    a.dim = d->dim;
    a.rot = positions ? d->rot : 0;
    a.max_pos = d->max_pos;
    a.interleaved = d->layout == FTCNN_ROPE_INTERLEAVED;
    a.weight_f32 = d->weight_dtype == FTCNN_F32;
    a.eps = d->eps;
    a.positions = positions;
    a.table = table;
    FT_PAGED_HIP(launch_rope(d->dtype, a, stream), what);
    return FTCNN_OK;
}

int ftcnn_kv_append(const ftcnn_append_desc *d, const void *k, const void *v, const int32_t *positions,
                    const float *table, const void *k_weight, const int64_t *slots, void *k_cache, void *v_cache,
                    hipStream_t stream) {
    const char *what = "kv_append";
    if (!d) return set_error(FTCNN_E_ARG, "%s: null descriptor", what);
    const int rc = check_rope(what, d->dtype, d->tokens, d->kv_heads, d->dim, d->rot, d->layout, d->max_pos, d->eps,
                              positions, table, k_weight != nullptr, d->weight_dtype);
    if (rc != FTCNN_OK) return rc;
    if (d->pages < 1 || d->page < 1)
        return set_error(FTCNN_E_SHAPE, "%s: %d pages of %d rows", what, d->pages, d->page);
    if (d->tokens == 0) return FTCNN_OK;
    if (!k || !v || !slots || !k_cache || !v_cache) return set_error(FTCNN_E_ARG, "%s: null pointer", what);
    RopeArgs a{};
    const void *in[2] = {k, v};
    void *out[2] = {k_cache, v_cache};
    const int64_t *is[2] = {d->k_stride, d->v_stride}, *os[2] = {d->k_cache_stride, d->v_cache_stride};
    for (int s = 0; s < 2; ++s) {
        a.x[1 + s] = in[s];
        a.y[1 + s] = out[s];
        a.heads[1 + s] = d->kv_heads;
        for (int i = 0; i < 3; ++i) {
            if (i < 2) a.xs[1 + s][i] = is[s][i];
            a.ys[1 + s][i] = os[s][i];
        }
    }
    a.weight[1] = k_weight;
    a.tokens = d->tokens;
    a.dim = d->dim;
    a.rot = positions ? d->rot : 0;
    a.max_pos = d->max_pos;
    a.interleaved = d->layout == FTCNN_ROPE_INTERLEAVED;
    a.weight_f32 = d->weight_dtype == FTCNN_F32;
    a.pages = d->pages;
    a.page = d->page;
    a.eps = d->eps;
    a.positions = positions;
    a.slots = slots;
    a.table = table;
    FT_PAGED_HIP(launch_rope(d->dtype, a, stream), what);
    return FTCNN_OK;
}

size_t ftcnn_paged_attention_workspace_bytes(const ftcnn_attention_desc *desc) {
    return check_attention(desc) == FTCNN_OK ? attn_plan(*desc).bytes : 0;
}

int ftcnn_paged_attention(const ftcnn_attention_desc *d, const void *q, const void *k_cache, const void *v_cache,
                          const int32_t *page_list, const int32_t *kv_lens, const int32_t *q_starts, void *out,
                          float *lse, void *workspace, hipStream_t stream) {
    const char *what = "paged_attention";
    const int rc = check_attention(d);
    if (rc != FTCNN_OK) return rc;
    if (!q_starts && d->tokens != d->batch)
        return set_error(FTCNN_E_SHAPE, "%s: %d tokens of %d sequences need q_starts", what, d->tokens, d->batch);
    if (d->tokens == 0) return FTCNN_OK;
    if (!out || (d->batch && (!q || !k_cache || !v_cache || !kv_lens || (!page_list && d->list_len))))
        return set_error(FTCNN_E_ARG, "%s: null pointer", what);
    const int vec = d->dtype == FTCNN_F32 ? 4 : 8;
    bool al = aligned16(q) && aligned16(k_cache) && aligned16(v_cache) && aligned16(out);
    for (int i = 0; i < 3; ++i) {
        if (i < 2) al = al && d->q_stride[i] % vec == 0 && d->out_stride[i] % vec == 0;
        al = al && d->k_cache_stride[i] % vec == 0 && d->v_cache_stride[i] % vec == 0;
        if (std::min(d->k_cache_stride[i], d->v_cache_stride[i]) < 0 ||
            std::max(d->k_cache_stride[i], d->v_cache_stride[i]) > kMaxRows / 2)
            return set_error(FTCNN_E_UNSUPPORTED, "%s: cache strides are 0 to 2^29 elements", what);
    }
    if (!al)
        return set_error(FTCNN_E_UNSUPPORTED, "%s: rows of q, out and the cache must start on 16 bytes", what);
    const AttnPlan pl = attn_plan(*d);
    if (pl.bytes && (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256))
        return set_error(FTCNN_E_WORKSPACE, "%s: workspace missing or not 256-byte aligned", what);
    const long long blocks = pl.groups ? pl.groups : (long long)pl.tiles * d->kv_heads * d->batch;
    if (blocks * attn_threads(pl) > kMaxThreads)
        return set_error(FTCNN_E_SHAPE, "%s: %lld workgroups", what, blocks);
    AttnArgs a{};
    a.q = q;
    a.k = k_cache;
    a.v = v_cache;
    a.o = out;
    a.lse = lse;
    if (pl.bytes) {
        char *ws = static_cast<char *>(workspace);
        a.part_o = reinterpret_cast<float *>(ws);
        a.part_ml = reinterpret_cast<float *>(ws + pl.part_ml);
        a.cuts = reinterpret_cast<AttnCut *>(ws + pl.cuts);
    }
    a.page_list = page_list;
    a.kv_lens = kv_lens;
    a.q_starts = q_starts;
    for (int i = 0; i < 3; ++i) {
        if (i < 2) {
            a.qs[i] = d->q_stride[i];
            a.os[i] = d->out_stride[i];
        }
        a.kb[i] = (unsigned)(d->k_cache_stride[i] * (16 / vec));
        a.vb[i] = (unsigned)(d->v_cache_stride[i] * (16 / vec));
    }
    a.list_stride = d->list_stride;
    a.batch = d->batch;
    a.tokens = d->tokens;
    a.kv_heads = d->kv_heads;
    a.group = d->heads / d->kv_heads;
    a.dim = d->dim;
    a.pages = d->pages;
    a.page = d->page;
    a.capacity = d->list_len * d->page;
    a.causal = d->causal != 0;
    // no sequence holds more than the list can name: a wider window hides nothing more, and sums of positions
    // and windows of at most 2^30 stay within 32 bits
    a.window = std::min(d->window, a.capacity);
    a.tiles = pl.tiles;
    a.groups = pl.groups;
    a.min_run = pl.min_run;
    a.unit_cost = pl.unit_cost;
    a.tile_keys = pl.keys;
    a.part_rows = pl.part_rows;
    a.interleave = pl.tiles > 1 && (long long)d->batch * d->kv_heads % 8 == 0;
    a.div_page = fast_div((uint32_t)d->page);
    a.div_group = fast_div((uint32_t)a.group);
    a.scale_log2 = d->scale * kLog2E;
    if (d->batch == 0) {
        FT_PAGED_HIP(launch_attn_clear(d->dtype, a, stream), what);
        return FTCNN_OK;
    }
    FT_PAGED_HIP(d->dtype == FTCNN_F32 ? launch_attn_f32(pl, a, stream) : launch_attn_bf16(pl, a, stream), what);
    if (pl.groups) FT_PAGED_HIP(launch_attn_join(d->dtype, pl, a, stream), "paged_attention: join");
    return FTCNN_OK;
}

}  // extern "C"
