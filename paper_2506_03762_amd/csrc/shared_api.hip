// Entry points of what stands around a prompt's cache: rotation by positions, the paged cache, the attention of a batch
// that shares prefixes, of packed prompts, of single tokens over paged caches, and the eviction from these.  All checks run on the host
// before anything is enqueued.
#include <math.h>

#include <algorithm>

#include "aha_host.h"

namespace aha {

constexpr double kLog2e = 1.4426950408889634;

// What the two kinds of geometry have in common.
static int32_t check_heads(int batch, int rows, const char *rows_name, int q_heads, int kv_heads, int d, int dtype) {
    if (batch < 1 || rows < 1 || q_heads < 1 || kv_heads < 1)
        return fail(AHA_ERR_INVALID_ARG, "batch, %s, n_q_heads and n_kv_heads must be >= 1", rows_name);
    if (dtype != AHA_F32 && dtype != AHA_BF16)
        return fail(AHA_ERR_INVALID_ARG, "dtype %d is neither AHA_F32 nor AHA_BF16", dtype);
    if (d != 64 && d != 128) return fail(AHA_ERR_UNSUPPORTED, "head_dim %d: only 64 and 128 are built", d);
    return AHA_OK;
}

// A written tensor: batches and heads a row or more apart (that the caller's axes do not overlap otherwise is up to them).
static int32_t check_out_stride(const char *name, const int64_t s[3], int64_t n0, int64_t n1, int dtype, int d) {
    const int32_t rc = check_stride(name, s, dtype, d);
    if (rc) return rc;
    if ((n0 > 1 && s[0] < d) || (n1 > 1 && s[1] < d))
        return fail(AHA_ERR_INVALID_ARG, "%s_stride: rows of what is written would overlap", name);
    return AHA_OK;
}

static int32_t check_rotary(const aha_rotary *p) {
    if (!p) return fail(AHA_ERR_INVALID_ARG, "params is null");
    const int32_t rc = check_heads(p->batch, p->tokens, "tokens", p->n_q_heads, p->n_kv_heads, p->head_dim, p->dtype);
    if (rc) return rc;
    // (up to 16 threads a row: a launch has fewer than 2^32)
    if ((int64_t)p->batch * p->tokens > 1 << 27) return fail(AHA_ERR_UNSUPPORTED, "batch * tokens beyond 2^27");
    if ((int64_t)p->n_q_heads + 2 * (int64_t)p->n_kv_heads > 65535)
        return fail(AHA_ERR_UNSUPPORTED, "n_q_heads + 2 n_kv_heads exceeds 65535");
    if (p->rot_dim < 0 || p->rot_dim > p->head_dim || p->rot_dim % 16 != 0)
        return fail(AHA_ERR_INVALID_ARG, "rot_dim (%d) must be a multiple of 16 in [0, head_dim]", p->rot_dim);
    if (p->pairing != AHA_PAIR_HALVES && p->pairing != AHA_PAIR_NEIGHBOURS)
        return fail(AHA_ERR_INVALID_ARG, "pairing %d is unknown", p->pairing);
    if (p->n_axes < 1 || p->n_axes > 4) return fail(AHA_ERR_INVALID_ARG, "n_axes (%d) must lie in [1, 4]", p->n_axes);
    if (p->transpose != 0 && p->transpose != 1) return fail(AHA_ERR_INVALID_ARG, "transpose must be 0 or 1");
    return AHA_OK;
}

static int32_t check_pages(const aha_pages *pg, int kv_heads, int dtype, int d, bool strides) {
    if (pg->n_pages < 1 || pg->table_width < 1)
        return fail(AHA_ERR_INVALID_ARG, "n_pages and table_width must be >= 1");
    if (pg->page_size < 1 || pg->page_size > 1024 || (pg->page_size & (pg->page_size - 1)))
        return fail(AHA_ERR_UNSUPPORTED, "page_size (%d) must be a power of two in [1, 1024]", pg->page_size);
    if (pg->n_pages > 1 << 30 || (int64_t)pg->table_width * pg->page_size > 1 << 30)
        return fail(AHA_ERR_UNSUPPORTED, "n_pages or table_width * page_size beyond 2^30");
    if (pg->reserved != 0) return fail(AHA_ERR_INVALID_ARG, "reserved must be 0");
    if (!strides) return AHA_OK;
    const int32_t rc = check_out_stride("pages.k", pg->k_stride, pg->n_pages, kv_heads, dtype, d);
    return rc ? rc : check_out_stride("pages.v", pg->v_stride, pg->n_pages, kv_heads, dtype, d);
}

static PageGeom page_geom(const aha_pages *pg, const int32_t *table, const int32_t *tail_len, const int32_t *new_len) {
    PageGeom g{};
    g.new_len = new_len;
    if (!pg) return g;
    for (int t = 0; t < 3; ++t) g.ks[t] = pg->k_stride[t], g.vs[t] = pg->v_stride[t];
    g.table = table;
    g.tail_len = tail_len;
    g.n_pages = pg->n_pages;
    g.page_shift = __builtin_ctz((unsigned)pg->page_size);
    g.table_width = pg->table_width;
    return g;
}

static RotaryGeom rotary_geom(const aha_rotary *p, const void *q, const void *k, const float *inv_freq, const int32_t *pair_axis,
                              const int32_t *positions, void *q_out) {
    RotaryGeom g{};
    g.q = q; g.k = k; g.q_out = q_out;
    for (int t = 0; t < 3; ++t) {
        g.qs[t] = p->q_stride[t]; g.ks[t] = p->k_stride[t]; g.vs[t] = p->v_stride[t];
        g.qo[t] = p->q_out_stride[t]; g.ko[t] = p->k_out_stride[t];
    }
    g.batch = p->batch; g.n = p->tokens; g.Hq = q ? p->n_q_heads : 0; g.Hkv = k ? p->n_kv_heads : 0;
    g.d = p->head_dim; g.dtype = p->dtype; g.rot = p->rot_dim; g.n_axes = p->n_axes;
    g.neighbours = p->pairing == AHA_PAIR_NEIGHBOURS; g.transpose = p->transpose != 0;
    g.inv_freq = inv_freq; g.pair_axis = pair_axis; g.positions = positions;
    return g;
}

// q with q_out, or neither; the angles' tables where something is turned.
static int32_t check_turned(const aha_rotary *p, const void *q, const void *q_out, const float *inv_freq, const int32_t *pair_axis,
                            const int32_t *positions) {
    int32_t rc;
    if ((q == nullptr) != (q_out == nullptr)) return fail(AHA_ERR_INVALID_ARG, "q and q_out must both be given or both be null");
    if (q && ((rc = check_ptr("q", q, 16)) || (rc = check_ptr("q_out", q_out, 16)) ||
              (rc = check_stride("q", p->q_stride, p->dtype, p->head_dim)) ||
              (rc = check_out_stride("q_out", p->q_out_stride, p->batch, p->n_q_heads, p->dtype, p->head_dim))))
        return rc;
    if (p->rot_dim > 0 && ((rc = check_ptr("inv_freq", inv_freq, 4)) || (rc = check_ptr("positions", positions, 4)) ||
                           (pair_axis && (rc = check_ptr("pair_axis", pair_axis, 4)))))
        return rc;
    return AHA_OK;
}

static int32_t check_shared(const aha_shared *p, const aha_pages *pg, bool strides) {
    if (!p) return fail(AHA_ERR_INVALID_ARG, "params is null");
    int32_t rc = check_heads(p->batch, p->q_len, "q_len", p->n_q_heads, p->n_kv_heads, p->head_dim, p->dtype);
    if (rc) return rc;
    if (p->n_q_heads % p->n_kv_heads != 0)
        return fail(AHA_ERR_INVALID_ARG, "n_q_heads (%d) is not a multiple of n_kv_heads (%d)", p->n_q_heads, p->n_kv_heads);
    const int64_t rows = (int64_t)(p->n_q_heads / p->n_kv_heads) * p->q_len;  // (each factor below 2^31)
    if ((int64_t)p->batch * p->n_kv_heads > 65535 || rows > 1 << 22 || rows * p->batch > 1 << 22)
        return fail(AHA_ERR_UNSUPPORTED, "batch * n_kv_heads exceeds 65535 or group * q_len * batch 2^22");
    if (p->n_prefixes < 0 || (p->n_prefixes > 0 && p->prefix_cap < 1))
        return fail(AHA_ERR_INVALID_ARG, "n_prefixes must be >= 0, prefix_cap >= 1");
    if (p->n_prefixes > 65535 || (p->n_prefixes > 0 && p->prefix_cap > 1 << 30))
        return fail(AHA_ERR_UNSUPPORTED, "n_prefixes exceeds 65535 or prefix_cap 2^30");
    if (!(p->scale >= 0.f) || isinf((float)(p->scale * kLog2e)))
        return fail(AHA_ERR_INVALID_ARG, "scale must be >= 0 and finite, times log2(e) too");
    if (p->reserved != 0) return fail(AHA_ERR_INVALID_ARG, "reserved must be 0");
    if (pg && (rc = check_pages(pg, p->n_kv_heads, p->dtype, p->head_dim, strides))) return rc;
    if (!strides) return AHA_OK;
    if ((rc = check_stride("q", p->q_stride, p->dtype, p->head_dim)) ||
        (rc = check_out_stride("out", p->out_stride, p->batch, p->n_q_heads, p->dtype, p->head_dim)))
        return rc;
    if (p->n_prefixes == 0) return AHA_OK;
    if ((rc = check_stride("k", p->k_stride, p->dtype, p->head_dim))) return rc;
    return check_stride("v", p->v_stride, p->dtype, p->head_dim);
}

// Rows of a tile for about `rows` rows that see the same keys.  us of a call with tiles of 32 and of 128 rows: 64 rows of 8 heads, 16384 keys
// 27.3, 36.2; 4 x 64 rows, 4096 keys, d = 64 34.8, 42.4; 128 rows of 8 heads 40.8, 44.1 for 16384 keys, 69.5, 58.1 for 32768; 128 rows of 32
// heads 124.8, 89.4; with tiles of 32 and of 256: 192 rows of 8 heads 60.2, 50.2.  Prefixes: the rows of an evenly filled one (which rows share
// which prefix is known on the device alone), so that calls with room for many prefixes take small tiles, however few are in use.
static int tile_rows(int dtype, int64_t rows) { return dtype != AHA_BF16 || rows <= 64 ? 32 : rows <= 128 ? 128 : 256; }
// Parts of an item's keys: as many as fill the chip (two workgroups per CU, large tiles one) with `tiles` in each, large tiles of four steps at
// least.
static int64_t parts_for(int64_t tiles, int64_t keys, int rows) {
    const int64_t step = rows > 32 ? 64 : 128, steps = (keys + step - 1) / step, resident = rows > 32 ? 256 : 512, least = rows > 32 ? 4 : 1;
    return std::max<int64_t>(1, std::min<int64_t>({(resident + tiles - 1) / tiles, (steps + least - 1) / least, 64}));
}
static SharedPlan plan_shared(const aha_shared *p, const aha_pages *pages) {
    SharedPlan pl{};
    const int64_t per = (int64_t)(p->n_q_heads / p->n_kv_heads) * p->q_len, all = per * p->batch;
    pl.tail_rows = tile_rows(p->dtype, per);
    pl.prefix_rows = pl.tail_rows;
    if (p->n_prefixes > 0) {
        pl.prefix_rows = tile_rows(p->dtype, all / p->n_prefixes);
        const int64_t tile = pl.prefix_rows, members = std::min<int64_t>(p->n_prefixes, p->batch);  // prefixes with rows, each with a tile that is not full
        const int64_t tiles = (all + members * (tile - 1)) / tile, parts = parts_for(tiles * p->n_kv_heads, p->prefix_cap, (int)tile);
        pl.prefix_tiles = (int)tiles;
        pl.prefix_parts = (int)parts;
        pl.prefix_items = (p->n_kv_heads * parts + 7) / 8 * 8 * tiles;
    }
    if (pages) {
        const int64_t tiles = (per + pl.tail_rows - 1) / pl.tail_rows, units = (int64_t)p->batch * p->n_kv_heads;
        const int64_t parts = parts_for(tiles * units, (int64_t)pages->table_width * pages->page_size, pl.tail_rows);
        pl.tail_tiles = (int)tiles;
        pl.tail_parts = (int)parts;
        pl.tail_items = (units * parts + 7) / 8 * 8 * tiles;
    }
    // (never 0, with which a masked logit, -inf, would be no number: a scale of 0 becomes the smallest subnormal, no logit then counts)
    pl.c_out = std::max((float)(p->scale * kLog2e), 0x1p-149f);
    const size_t rows = (size_t)all * p->n_kv_heads * (pl.prefix_parts + pl.tail_parts);
    pl.off_ms = align_up(sizeof(float) * rows * p->head_dim, 256);
    pl.bytes = align_up(pl.off_ms + 2 * sizeof(float) * rows, 256);
    return pl;
}

// (workgroups of 256 threads: a launch has fewer than 2^32)
static int32_t check_items(const SharedPlan &pl) {
    if (pl.prefix_items + pl.tail_items > 1 << 23)
        return fail(AHA_ERR_UNSUPPORTED, "problem exceeds the launch grid limits");
    return AHA_OK;
}

// Two strides of rows whose head_dim channels are contiguous, as check_stride() has them.
static int32_t check_pair(const char *name, const int64_t s[2], int dtype, int d, bool out, int64_t n0, int64_t n1) {
    const int a = 16 / esize(dtype);
    for (int t = 0; t < 2; ++t) {
        const int64_t n = t ? n1 : n0;
        if (s[t] < 0 || s[t] % a != 0)
            return fail(AHA_ERR_INVALID_ARG, "%s_stride[%d]=%lld must be a non-negative multiple of %d elements", name, t, (long long)s[t], a);
        if (out && n > 1 && s[t] < d) return fail(AHA_ERR_INVALID_ARG, "%s_stride: rows of what is written would overlap", name);
    }
    return AHA_OK;
}
static int32_t check_scale(const char *name, float scale) {
    if (!(scale >= 0.f) || isinf((float)(scale * kLog2e)))
        return fail(AHA_ERR_INVALID_ARG, "%s must be >= 0 and finite, times log2(e) too", name);
    return AHA_OK;
}
// (never 0, with which a masked logit, -inf, would be no number: a scale of 0 becomes the smallest subnormal, no logit then counts)
static float log2_scale(float scale) { return std::max((float)(scale * kLog2e), 0x1p-149f); }

static int32_t check_prompt(const aha_prompt *p, bool strides) {
    if (!p) return fail(AHA_ERR_INVALID_ARG, "params is null");
    int32_t rc = check_heads(p->sequences, p->tokens, "tokens", p->n_q_heads, p->n_kv_heads, p->head_dim, p->dtype);
    if (rc) return rc;
    if (p->n_q_heads % p->n_kv_heads != 0)
        return fail(AHA_ERR_INVALID_ARG, "n_q_heads (%d) is not a multiple of n_kv_heads (%d)", p->n_q_heads, p->n_kv_heads);
    // (a tile has a row at least, and the numbers of the tiles of 16 and 32 rows are rounded up to a group of eight: fewer than 2^31)
    if (p->sequences > 65535 || p->n_kv_heads > 65535 || (int64_t)p->tokens * p->n_q_heads > 1 << 30 || p->n_q_heads / p->n_kv_heads > 1 << 25)
        return fail(AHA_ERR_UNSUPPORTED, "sequences or n_kv_heads exceeds 65535, tokens * n_q_heads 2^30 or n_q_heads / n_kv_heads 2^25");
    if ((rc = check_scale("scale", p->scale))) return rc;
    if (p->reserved != 0) return fail(AHA_ERR_INVALID_ARG, "reserved must be 0");
    if (!strides) return AHA_OK;
    if ((rc = check_pair("q", p->q_stride, p->dtype, p->head_dim, false, 0, 0)) ||
        (rc = check_pair("k", p->k_stride, p->dtype, p->head_dim, false, 0, 0)) ||
        (rc = check_pair("v", p->v_stride, p->dtype, p->head_dim, false, 0, 0)))
        return rc;
    return check_pair("out", p->out_stride, p->dtype, p->head_dim, true, p->tokens, p->n_q_heads);
}

// What a tile of the attention of packed prompts costs, us: its start and end, 32 keys of it, and by how much those that do not run at once with the first
// ones cost more.
struct PromptTiles {
    int rows, unit, slots;  // rows; of one head at a time; tiles that run at once
    float start, block, later;
};
static PromptPlan plan_prompt(const aha_prompt *p) {
    PromptPlan pl{};
    // The cheapest tiles by an estimate for prompts of equal lengths (the host knows no others): the first ones' cost, all of a prompt's keys, and the average
    // one's for every further round.  The numbers are fitted to the times of 324 shapes (1 to 64 prompts of 20 to 8192 tokens, 2 to 64 heads): what they
    // choose is 0.8 % (d = 64 0.1) slower than the fastest tiles on average, and 1.2 times at worst (one prompt of 8192, 6 heads over 2: 178, 173, 206 us in the
    // order of the table).  d = 128, 32 heads over 8: one prompt of 512 13.5, 16.0, 21.9, 1024 31.1, 26.8, 34.8, 4096 241, 146, 135, 16 of 200 55, 23.5,
    // 32; 8 over 2: one of 2048 29.2, 45, 58, 16 of 64 7.6, 6.8, 10.2.  d = 64, 16 heads: one of 1024 12.4, 20.4, 28.5, of 4096 71, 70, 88, 16 of 500
    // 42.5, 27.1, 28.6.
    // fp32, 300 shapes: 1.0 and 0.6 % (1.15 and 1.4 times: 16 prompts of 20 tokens, 16 heads, 8.0, 10.9 in the order of the table).  d = 64: one prompt of 512, 2
    // heads, 10.7, 16.0, 8 heads of 2048 71, 69, of 4096 245, 191; d = 128: 2 heads of 1024 28.9, 43.9, 8 of 1024 56, 47.
    static constexpr PromptTiles kTiles[2][3] = {
        {{32, 32, 512, 5.84f, .17f, 1.14f}, {128, 32, 512, 5.11f, .5f, 1.27f}, {256, 64, 256, 6.31f, .52f, 1.16f}},  // d = 64
        {{32, 32, 512, 8.86f, .35f, 1.f}, {128, 32, 512, 7.73f, .6f, 1.14f}, {256, 64, 256, 15.34f, .57f, .92f}}};   // d = 128
    const int64_t prompts = std::min<int64_t>(p->sequences, p->tokens), group = p->n_q_heads / p->n_kv_heads, n = (p->tokens + prompts - 1) / prompts;
    static constexpr PromptTiles kTilesF32[2][2] = {{{16, 16, 256, 4.11f, .6f, .48f}, {32, 32, 256, 6.55f, .72f, .68f}},    // d = 64
                                                    {{16, 16, 256, 5.41f, 1.18f, .67f}, {32, 32, 256, 9.29f, 1.15f, .73f}}};  // d = 128
    float least = INFINITY;
    auto try_tiles = [&](const PromptTiles &t) {
        if (p->tokens / t.rows > 1 << 25) return;  // (tile_of() counts fewer than 2^26 tiles to a prompt: 16 rows, 2^29 tokens)
        const int64_t units = (n + t.unit - 1) / t.unit * group, heads = t.rows / t.unit;  // (a tile of 32 rows: one unit)
        const int64_t tiles = prompts * ((units + heads - 1) / heads) * p->n_kv_heads;
        const float keys = t.block * (float)n / 32;
        const float time = t.start + keys + std::max(0.f, (float)tiles / t.slots - 1.f) * t.later * (t.start + keys / 2);
        if (time >= least) return;
        least = time;
        pl.rows = t.rows;
        pl.staged = tiles > 256;  // (more than one workgroup to a CU: over 162 shapes 0.4 % slower than the faster one on average; never 6, always 0.9)
        // at most: one unit's rows, and one tile, of every prompt are not full
        pl.items = ((p->tokens + (t.unit - 1) * prompts) / t.unit * group + prompts * (heads - 1)) / heads * p->n_kv_heads;
        if (heads == 1) pl.items = (pl.items / group + 7) / 8 * 8 * group;
    };
    if (p->dtype == AHA_BF16)
        for (const PromptTiles &t : kTiles[p->head_dim == 128]) try_tiles(t);
    else
        for (const PromptTiles &t : kTilesF32[p->head_dim == 128]) try_tiles(t);
    return pl;
}

// What the attention of single tokens and the eviction have in common.
static int32_t check_paged(const aha_paged *p, const aha_pages *pg, int q_heads, int least_slots, bool strides) {
    if (!p) return fail(AHA_ERR_INVALID_ARG, "params is null");
    if (!pg) return fail(AHA_ERR_INVALID_ARG, "pages is null");
    int32_t rc = check_heads(p->batch, 1, "batch", q_heads, p->n_kv_heads, p->head_dim, p->dtype);
    if (rc) return rc;
    if ((int64_t)p->batch * p->n_kv_heads > 65535) return fail(AHA_ERR_UNSUPPORTED, "batch * n_kv_heads exceeds 65535");
    if (p->slots < least_slots) return fail(AHA_ERR_INVALID_ARG, "slots (%d) must be >= %d", p->slots, least_slots);
    if (p->slots > 1 << 30) return fail(AHA_ERR_UNSUPPORTED, "slots beyond 2^30");
    if (p->budget < 1) return fail(AHA_ERR_INVALID_ARG, "budget (%d) must be >= 1", p->budget);
    if (p->reserved != 0) return fail(AHA_ERR_INVALID_ARG, "reserved must be 0");
    return check_pages(pg, p->n_kv_heads, p->dtype, p->head_dim, strides);
}
// Rows of `slots` numbers.
static int32_t check_slots(const char *name, const int64_t s[2], const aha_paged *p, bool out) {
    const int64_t n[2] = {p->batch, p->n_kv_heads};
    for (int t = 0; t < 2; ++t) {
        if (s[t] < 0) return fail(AHA_ERR_INVALID_ARG, "%s_stride[%d] is negative", name, t);
        if (out && n[t] > 1 && s[t] < p->slots) return fail(AHA_ERR_INVALID_ARG, "%s_stride: rows of what is written would overlap", name);
    }
    return AHA_OK;
}

static int32_t check_paged_attention(const aha_paged *p, const aha_pages *pg, bool strides) {
    int32_t rc = check_paged(p, pg, p ? p->n_q_heads : 1, 0, strides);
    if (rc) return rc;
    if (p->n_q_heads % p->n_kv_heads != 0)
        return fail(AHA_ERR_INVALID_ARG, "n_q_heads (%d) is not a multiple of n_kv_heads (%d)", p->n_q_heads, p->n_kv_heads);
    if (p->n_q_heads / p->n_kv_heads > 1024 || (int64_t)p->batch * p->n_q_heads > 1 << 22)
        return fail(AHA_ERR_UNSUPPORTED, "n_q_heads / n_kv_heads exceeds 1024 or batch * n_q_heads 2^22");
    if (p->scale_mode != AHA_SCALE_FIXED && p->scale_mode != AHA_SCALE_ADAPTIVE)
        return fail(AHA_ERR_INVALID_ARG, "scale_mode %d is unknown", p->scale_mode);
    if ((rc = check_scale("scale", p->scale)) || (rc = check_scale("fixed_scale", p->fixed_scale))) return rc;
    if (!isfinite((float)(p->lambda_floor * kLog2e))) return fail(AHA_ERR_INVALID_ARG, "lambda_floor must be finite, times log2(e) too");
    if (!strides) return AHA_OK;
    if ((rc = check_pair("q", p->q_stride, p->dtype, p->head_dim, false, 0, 0))) return rc;
    return check_pair("out", p->out_stride, p->dtype, p->head_dim, true, p->batch, p->n_q_heads);
}

static PagedPlan plan_paged(const aha_paged *p, const aha_pages *pages) {
    PagedPlan pl{};
    const int group = p->n_q_heads / p->n_kv_heads;
    const int64_t units = (int64_t)p->batch * p->n_kv_heads;
    int64_t room = (int64_t)pages->table_width * pages->page_size;
    if (p->slots > 0) room = std::min<int64_t>(room, p->slots);
    // (fp32: tiles of 32 rows that are half empty take 1.2 to 1.5 times as long: d = 128 (64), 8 caches of 400 tokens, 8 x 4 heads 19.5, so 15.4 us (13.1, 11.3),
    // 64 of 1000, 8 x 1 heads 130, 107 (59, 47))
    pl.rows = p->dtype == AHA_F32 && group <= 16 ? 16 : 32;
    pl.tiles = (group + pl.rows - 1) / pl.rows;
    // (no part of more than 1024 places: sequences' lengths differ.  64 of up to 4096 tokens, 8 heads: 168 us with one part each, 160 with four, 167 with
    // eight)
    pl.parts = (int)std::max(parts_for(units * pl.tiles, room, 32), std::min<int64_t>(64, room / 1024));
    // (workgroups of 256 threads: a launch has fewer than 2^32.  At most 2^22 rows in 65535 (sequence, KV head) pairs: 43 parts at least)
    pl.parts = (int)std::min<int64_t>(pl.parts, (1 << 23) / (units * pl.tiles));
    // One launch where parts would shorten the chain of a sequence's blocks by less than the second one takes.  us with parts and in one, d = 128 (64), 64
    // (sequence, KV head) pairs, 4 query heads each: 256 tokens 12.0, 10.5 (10.9, 8.9), 384 12.2, 13.0 (11.1, 9.9), 768 15.3, 17.9 (13.2, 13.2); 128 pairs: 512
    // 16.3, 15.1 (13.6, 11.6), 768 20.9, 19.0 (15.7, 13.7), 1000 22.8, 23.0 (16.3, 16.0); 512 pairs of 400, which are never split, 29.9, 24.0; fp32, whose
    // blocks take longer, 64 pairs of 256 13.8, 14.3 (11.3, 10.2), 128 pairs of 768 31.8, 28.9 (21.5, 19.2), in tiles of 32 rows 64 pairs of 256 16.9, 20.1 (12.8,
    // 13.1).
    const int64_t blocks = (room + 127) / 128, saved = blocks - (blocks + pl.parts - 1) / pl.parts;
    const bool bf16 = p->dtype == AHA_BF16;
    pl.one = pl.tiles == 1 && saved <= (!bf16 && pl.rows > 16 ? 0 : units >= 128 ? 4 : p->head_dim == 64 ? (bf16 ? 3 : 1) : (bf16 ? 1 : 0));
    if (pl.one) pl.parts = 1;
    pl.items = units * pl.tiles * pl.parts;
    pl.ld = p->slots > 0 ? (room + 31) / 32 * 32 : 0;
    const size_t rows = (size_t)units * group;
    if (!pl.one) {
        pl.off_ms = align_up(sizeof(float) * rows * pl.parts * p->head_dim, 256);
        pl.off_ms2 = align_up(pl.off_ms + 2 * sizeof(float) * rows * pl.parts, 256);
        pl.off_dots = align_up(pl.off_ms2 + 2 * sizeof(float) * rows * pl.parts, 256);
    }
    pl.bytes = align_up(pl.off_dots + sizeof(float) * rows * (size_t)pl.ld, 256);
    return pl;
}

static int32_t check_evict(const aha_paged *p, const aha_pages *pg, bool strides) {
    const int32_t rc = check_paged(p, pg, 1, 1, strides);
    if (rc) return rc;
    if (p->recent < 0 || p->sink < 0 || (int64_t)p->recent + p->sink > p->budget)
        return fail(AHA_ERR_INVALID_ARG, "recent (%d) and sink (%d) must be >= 0, together at most budget (%d)", p->recent, p->sink, p->budget);
    return AHA_OK;
}
static EvictPlan plan_evict(const aha_paged *p, const aha_pages *pages) {
    EvictPlan pl{};
    const int64_t room = std::min<int64_t>((int64_t)pages->table_width * pages->page_size, p->slots);
    const int64_t units = (int64_t)p->batch * p->n_kv_heads;
    pl.moves = (int)std::max<int64_t>(0, std::min<int64_t>(p->budget, room - p->budget));
    // keys of as many tokens as there can be or as fit, of the places that fill the last step of every wave, and 16 bits for each place that
    // becomes free (as many as tokens lie behind it, at most) and each that moves
    pl.waves = room <= 1024 ? 4 : room <= 4096 ? 8 : 16;
    const int64_t words = (int64_t)kEvictDynamic / 4 - 64 * pl.waves - 4;
    pl.lds_tokens = (int)std::min<int64_t>(room, std::max<int64_t>(words - pl.moves, words * 2 / 3));
    pl.lds_bytes = align_up(4 * ((size_t)pl.lds_tokens + 64 * pl.waves + std::min(pl.moves, pl.lds_tokens / 2)), 16);
    pl.in_one = pl.moves <= 256;
    pl.off_moves = align_up(sizeof(int32_t) * units, 256);
    pl.bytes = align_up(pl.off_moves + 2 * sizeof(int32_t) * (size_t)units * pl.moves, 256);
    return pl;
}

}  // namespace aha

using namespace aha;

extern "C" {

int32_t aha_rotate(const aha_rotary *p, const void *q, const void *k, const float *inv_freq, const int32_t *pair_axis,
                   const int32_t *positions, void *q_out, void *k_out, void *stream) {
    int32_t rc = check_rotary(p);
    if (rc) return rc;
    if (!q && !k) return fail(AHA_ERR_INVALID_ARG, "q and k are both null");
    if ((k == nullptr) != (k_out == nullptr)) return fail(AHA_ERR_INVALID_ARG, "k and k_out must both be given or both be null");
    if ((rc = check_turned(p, q, q_out, inv_freq, pair_axis, positions))) return rc;
    if (k && ((rc = check_ptr("k", k, 16)) || (rc = check_ptr("k_out", k_out, 16)) ||
              (rc = check_stride("k", p->k_stride, p->dtype, p->head_dim)) ||
              (rc = check_out_stride("k_out", p->k_out_stride, p->batch, p->n_kv_heads, p->dtype, p->head_dim))))
        return rc;
    RotaryGeom g = rotary_geom(p, q, k, inv_freq, pair_axis, positions, q_out);
    g.k_out = k_out;
    return hip_result(launch_rotate(g, (hipStream_t)stream), "rotation kernel");
}

int32_t aha_append_paged(const aha_rotary *p, const aha_pages *pages, const void *q, const void *k, const void *v,
                         const float *inv_freq, const int32_t *pair_axis, const int32_t *positions, const int32_t *page_table,
                         const int32_t *tail_len, const int32_t *new_len, void *q_out, void *k_pages, void *v_pages,
                         void *stream) {
    int32_t rc = check_rotary(p);
    if (rc) return rc;
    if (!pages) return fail(AHA_ERR_INVALID_ARG, "pages is null");
    if ((rc = check_pages(pages, p->n_kv_heads, p->dtype, p->head_dim, true)) ||
        (rc = check_turned(p, q, q_out, inv_freq, pair_axis, positions)))
        return rc;
    if ((rc = check_ptr("k", k, 16)) || (rc = check_ptr("v", v, 16)) || (rc = check_ptr("k_pages", k_pages, 16)) ||
        (rc = check_ptr("v_pages", v_pages, 16)) || (rc = check_ptr("page_table", page_table, 4)) ||
        (rc = check_ptr("tail_len", tail_len, 4)) || (new_len && (rc = check_ptr("new_len", new_len, 4))) ||
        (rc = check_stride("k", p->k_stride, p->dtype, p->head_dim)) ||
        (rc = check_stride("v", p->v_stride, p->dtype, p->head_dim)))
        return rc;
    RotaryGeom g = rotary_geom(p, q, k, inv_freq, pair_axis, positions, q_out);
    g.append = true;
    g.v = v;
    g.k_out = k_pages;
    g.v_out = v_pages;
    g.pages = page_geom(pages, page_table, tail_len, new_len);
    return hip_result(launch_rotate(g, (hipStream_t)stream), "append kernel");
}

int32_t aha_shared_attention_workspace_bytes(const aha_shared *p, const aha_pages *pages, size_t *out_bytes) {
    if (!out_bytes) return fail(AHA_ERR_INVALID_ARG, "out_bytes is null");
    int32_t rc = check_shared(p, pages, false);
    if (rc) return rc;
    const SharedPlan pl = plan_shared(p, pages);
    if ((rc = check_items(pl))) return rc;
    *out_bytes = pl.bytes;
    return AHA_OK;
}

int32_t aha_shared_attention(const aha_shared *p, const aha_pages *pages, const void *q, const void *k_prefix, const void *v_prefix,
                             const int32_t *prefix_len, const int32_t *prefix_first, const void *k_pages, const void *v_pages,
                             const int32_t *page_table, const int32_t *tail_len, const int32_t *new_len, void *out, float *lse,
                             void *workspace, size_t workspace_bytes, void *stream) {
    int32_t rc = check_shared(p, pages, true);
    if (rc) return rc;
    if ((rc = check_ptr("q", q, 16)) || (rc = check_ptr("out", out, 16)) || (lse && (rc = check_ptr("lse", lse, 4))) ||
        (new_len && (rc = check_ptr("new_len", new_len, 4))))
        return rc;
    if (p->n_prefixes > 0 && ((rc = check_ptr("k_prefix", k_prefix, 16)) || (rc = check_ptr("v_prefix", v_prefix, 16)) ||
                              (rc = check_ptr("prefix_len", prefix_len, 4)) || (rc = check_ptr("prefix_first", prefix_first, 4))))
        return rc;
    if (pages) {
        if ((rc = check_ptr("k_pages", k_pages, 16)) || (rc = check_ptr("v_pages", v_pages, 16)) ||
            (rc = check_ptr("page_table", page_table, 4)) || (rc = check_ptr("tail_len", tail_len, 4)))
            return rc;
    } else if (k_pages || v_pages || page_table || tail_len) {
        return fail(AHA_ERR_INVALID_ARG, "pages is null, but tails are given");
    }
    const SharedPlan pl = plan_shared(p, pages);
    if ((rc = check_items(pl))) return rc;
    if ((rc = check_ws(workspace, workspace_bytes, pl.bytes))) return rc;
    SharedGeom g{};
    g.q = q; g.kp = k_prefix; g.vp = v_prefix; g.kt = k_pages; g.vt = v_pages; g.out = out; g.lse = lse;
    g.prefix_len = prefix_len; g.prefix_first = prefix_first;
    for (int t = 0; t < 3; ++t) {
        g.qs[t] = p->q_stride[t]; g.os[t] = p->out_stride[t]; g.ks[t] = p->k_stride[t]; g.vs[t] = p->v_stride[t];
    }
    g.pages = page_geom(pages, page_table, tail_len, new_len);
    g.batch = p->batch; g.n = p->q_len; g.Hq = p->n_q_heads; g.Hkv = p->n_kv_heads; g.G = g.Hq / g.Hkv;
    g.d = p->head_dim; g.dtype = p->dtype; g.n_prefixes = p->n_prefixes; g.prefix_cap = p->prefix_cap;
    return hip_result(launch_shared_attention(g, pl, workspace, (hipStream_t)stream), "shared-prefix attention kernels");
}

int32_t aha_prompt_attention_workspace_bytes(const aha_prompt *p, size_t *out_bytes) {
    if (!out_bytes) return fail(AHA_ERR_INVALID_ARG, "out_bytes is null");
    const int32_t rc = check_prompt(p, false);
    if (rc) return rc;
    *out_bytes = 0;
    return AHA_OK;
}

int32_t aha_prompt_attention_tile_rows(const aha_prompt *p, int32_t *out_rows) {
    if (!out_rows) return fail(AHA_ERR_INVALID_ARG, "out_rows is null");
    const int32_t rc = check_prompt(p, false);
    if (rc) return rc;
    *out_rows = plan_prompt(p).rows;
    return AHA_OK;
}

int32_t aha_prompt_attention(const aha_prompt *p, const void *q, const void *k, const void *v, const int32_t *first, void *out, float *lse,
                             void *workspace, size_t workspace_bytes, void *stream) {
    int32_t rc = check_prompt(p, true);
    if (rc) return rc;
    if ((rc = check_ptr("q", q, 16)) || (rc = check_ptr("k", k, 16)) || (rc = check_ptr("v", v, 16)) || (rc = check_ptr("out", out, 16)) ||
        (rc = check_ptr("first", first, 4)) || (lse && (rc = check_ptr("lse", lse, 4))))
        return rc;
    const PromptPlan pl = plan_prompt(p);
    if ((rc = check_ws(workspace, workspace_bytes, 0))) return rc;
    PromptGeom g{};
    g.q = q; g.k = k; g.v = v; g.out = out; g.lse = lse; g.first = first;
    for (int t = 0; t < 2; ++t) {
        g.qs[t] = p->q_stride[t]; g.ks[t] = p->k_stride[t]; g.vs[t] = p->v_stride[t]; g.os[t] = p->out_stride[t];
    }
    g.tokens = p->tokens; g.sequences = p->sequences; g.Hq = p->n_q_heads; g.Hkv = p->n_kv_heads; g.G = g.Hq / g.Hkv;
    g.d = p->head_dim; g.dtype = p->dtype; g.c_out = log2_scale(p->scale);
    return hip_result(launch_prompt_attention(g, pl, (hipStream_t)stream), "prompt attention kernel");
}

int32_t aha_paged_attention_workspace_bytes(const aha_paged *p, const aha_pages *pages, size_t *out_bytes) {
    if (!out_bytes) return fail(AHA_ERR_INVALID_ARG, "out_bytes is null");
    const int32_t rc = check_paged_attention(p, pages, false);
    if (rc) return rc;
    *out_bytes = plan_paged(p, pages).bytes;
    return AHA_OK;
}

int32_t aha_paged_attention(const aha_paged *p, const aha_pages *pages, const void *q, const void *k_pages, const void *v_pages,
                            const int32_t *page_table, const int32_t *tail_len, const int32_t *seen, float *scores, int32_t *pos, void *out,
                            float *lse, void *workspace, size_t workspace_bytes, void *stream) {
    int32_t rc = check_paged_attention(p, pages, true);
    if (rc) return rc;
    if ((rc = check_ptr("q", q, 16)) || (rc = check_ptr("k_pages", k_pages, 16)) || (rc = check_ptr("v_pages", v_pages, 16)) ||
        (rc = check_ptr("page_table", page_table, 4)) || (rc = check_ptr("tail_len", tail_len, 4)) ||
        (seen && (rc = check_ptr("seen", seen, 4))) || (rc = check_ptr("out", out, 16)) || (lse && (rc = check_ptr("lse", lse, 4))))
        return rc;
    if (p->slots == 0 && (scores || pos)) return fail(AHA_ERR_INVALID_ARG, "slots is 0, but scores or pos are given");
    if (p->slots > 0 && ((rc = check_ptr("scores", scores, 4)) || (rc = check_slots("scores", p->scores_stride, p, true)) ||
                         (pos && ((rc = check_ptr("pos", pos, 4)) || (rc = check_slots("pos", p->pos_stride, p, true))))))
        return rc;
    const PagedPlan pl = plan_paged(p, pages);
    if ((rc = check_ws(workspace, workspace_bytes, pl.bytes))) return rc;
    PagedGeom g{};
    g.q = q; g.kt = k_pages; g.vt = v_pages; g.out = out; g.lse = lse; g.scores = scores; g.pos = pos; g.seen = seen;
    for (int t = 0; t < 2; ++t) {
        g.qs[t] = p->q_stride[t]; g.os[t] = p->out_stride[t]; g.ss[t] = p->scores_stride[t]; g.ps[t] = p->pos_stride[t];
    }
    g.pages = page_geom(pages, page_table, tail_len, nullptr);
    g.batch = p->batch; g.Hq = p->n_q_heads; g.Hkv = p->n_kv_heads; g.G = g.Hq / g.Hkv; g.d = p->head_dim; g.dtype = p->dtype;
    g.slots = p->slots; g.budget = p->budget; g.scale_mode = p->scale_mode;
    g.c_out = log2_scale(p->scale); g.fixed_scale = p->fixed_scale; g.lambda_floor = p->lambda_floor;
    return hip_result(launch_paged_attention(g, pl, workspace, (hipStream_t)stream), "paged attention kernels");
}

int32_t aha_paged_evict_workspace_bytes(const aha_paged *p, const aha_pages *pages, size_t *out_bytes) {
    if (!out_bytes) return fail(AHA_ERR_INVALID_ARG, "out_bytes is null");
    const int32_t rc = check_evict(p, pages, false);
    if (rc) return rc;
    *out_bytes = plan_evict(p, pages).bytes;
    return AHA_OK;
}

int32_t aha_paged_evict(const aha_paged *p, const aha_pages *pages, const float *scores, const int32_t *pos, void *k_pages, void *v_pages,
                        const int32_t *page_table, const int32_t *tail_len, const int32_t *seen, float *scores_out, int32_t *pos_out,
                        int32_t *len_out, void *workspace, size_t workspace_bytes, void *stream) {
    int32_t rc = check_evict(p, pages, true);
    if (rc) return rc;
    if ((rc = check_ptr("scores", scores, 4)) || (pos && (rc = check_ptr("pos", pos, 4))) || (rc = check_ptr("k_pages", k_pages, 16)) ||
        (rc = check_ptr("v_pages", v_pages, 16)) || (rc = check_ptr("page_table", page_table, 4)) || (rc = check_ptr("tail_len", tail_len, 4)) ||
        (seen && (rc = check_ptr("seen", seen, 4))) || (rc = check_ptr("scores_out", scores_out, 4)) ||
        (rc = check_ptr("pos_out", pos_out, 4)) || (rc = check_ptr("len_out", len_out, 4)) ||
        (rc = check_slots("scores", p->scores_stride, p, false)) || (pos && (rc = check_slots("pos", p->pos_stride, p, false))) ||
        (rc = check_slots("scores_out", p->scores_out_stride, p, true)) || (rc = check_slots("pos_out", p->pos_out_stride, p, true)))
        return rc;
    if (len_out == tail_len || len_out == seen) return fail(AHA_ERR_INVALID_ARG, "len_out is tail_len or seen, which other workgroups still read");
    auto other_rows = [&](const int64_t a[2], const int64_t b[2]) {
        return (p->batch > 1 && a[0] != b[0]) || (p->n_kv_heads > 1 && a[1] != b[1]);
    };
    if ((scores_out == scores && other_rows(p->scores_stride, p->scores_out_stride)) ||
        (pos_out == pos && other_rows(p->pos_stride, p->pos_out_stride)))
        return fail(AHA_ERR_INVALID_ARG, "in place, scores and scores_out, or pos and pos_out, must have the same strides");
    const EvictPlan pl = plan_evict(p, pages);
    if ((rc = check_ws(workspace, workspace_bytes, pl.bytes))) return rc;
    EvictGeom g{};
    g.scores = scores; g.pos = pos; g.seen = seen; g.kt = k_pages; g.vt = v_pages;
    g.scores_out = scores_out; g.pos_out = pos_out; g.len_out = len_out;
    for (int t = 0; t < 2; ++t) {
        g.ss[t] = p->scores_stride[t]; g.ps[t] = p->pos_stride[t]; g.so[t] = p->scores_out_stride[t]; g.po[t] = p->pos_out_stride[t];
    }
    g.pages = page_geom(pages, page_table, tail_len, nullptr);
    g.batch = p->batch; g.Hkv = p->n_kv_heads; g.d = p->head_dim; g.dtype = p->dtype; g.slots = p->slots; g.budget = p->budget;
    g.recent = p->recent; g.sink = p->sink;
    return hip_result(launch_paged_evict(g, pl, workspace, (hipStream_t)stream), "eviction kernels");
}

}  // extern "C"
