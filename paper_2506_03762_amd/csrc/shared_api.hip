// Entry points of what stands around a prompt's cache: rotation by positions, the paged cache, the attention of a batch
// that shares prefixes.  All checks run on the host before anything is enqueued.
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

}  // extern "C"
