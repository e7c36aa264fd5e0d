// What the kernels of the attention behind shared prefixes have in common: which rows and keys a workgroup takes, where a
// row and a key lie, the partial outputs in the workspace.
//
// The rows of a KV head are those of all sequences, query heads of its group and new tokens, one behind the other: row (b, gi, t)
// is number (b G + gi) n + t.  So the rows of a prefix are consecutive, as its sequences are.  A work item is a tile of
// consecutive rows and a range of keys: either of rows that share a prefix, over its keys, or of the rows of one sequence, over its
// tail.  Its result, relative to a reference of its own, goes to the workspace under the row's number and its part's; another launch joins a
// row's parts.
#pragma once

#include "key_places.h"

namespace aha {

struct SharedItem {
    bool prefix;     // else a tail
    int which;       // the prefix, or the sequence
    int h, part;     // KV head; number of the row's part
    int row0, row1;  // rows [row0, row1), row1 - row0 at most a tile
    int begin, end;  // keys; begin >= end: none
};

// first sequence of prefix g, within the batch
__device__ __forceinline__ int first_of(const SharedGeom &g, int i) { return min(max(g.prefix_first[i], 0), g.batch); }
__device__ __forceinline__ int rows_of_sequence(const SharedGeom &g) { return g.G * g.n; }
__device__ __forceinline__ int fresh_of(const SharedGeom &g, int b) {
    return g.pages.new_len ? min(max(g.pages.new_len[b], 0), g.n) : g.n;
}

// The prefix whose tile number `tile` is (tiles are counted prefix by prefix): its first and last sequence and its length; `tile` becomes the
// number among its own.  -1: there are fewer tiles.  64 prefixes at a time, one per lane, so that all that a work item has to
// know comes with one round of loads; all lanes of a wave call it and get the same.
__device__ __forceinline__ int prefix_of_tile(const SharedGeom &g, int rows, int lane, int &tile, int &first, int &end, int &len) {
    const int per = rows_of_sequence(g);
    for (int base = 0; base < g.n_prefixes; base += 64) {
        const int i = base + lane;
        int lo = 0, hi = 0, n = 0;
        if (i < g.n_prefixes) lo = first_of(g, i), hi = first_of(g, i + 1), n = min(max(g.prefix_len[i], 0), g.prefix_cap);
        const int tiles = (max(0, hi - lo) * per + rows - 1) / rows;
        int sum = tiles;  // over the lanes up to this one
#pragma unroll
        for (int s = 1; s < 64; s *= 2) {
            const int x = __shfl_up(sum, s);
            if (lane >= s) sum += x;
        }
        const uint64_t beyond = __builtin_amdgcn_ballot_w64(sum > tile);
        if (beyond) {
            const int at = __builtin_ctzll(beyond);
            tile -= __shfl(sum - tiles, at);
            first = __shfl(lo, at);
            end = __shfl(hi, at);
            len = __shfl(n, at);
            return base + at;
        }
        tile -= __shfl(sum, 63);
    }
    return -1;
}

// Work item of workgroup `id`: the tails' items first, whose lengths differ most (64 sequences of four prefixes of 4096 tokens 63.3 us
// with the prefixes' first, so 59.5).  Items of the same keys get numbers that are congruent modulo the XCDs, whose
// workgroups share an L2.  `rows`: of a tile; `step`: keys that ranges are multiples of.  false: nothing to do.
__device__ __forceinline__ bool shared_item(const SharedGeom &g, const SharedPlan &pl, int id, int rows, int step, int lane,
                                            SharedItem &it) {
    it.prefix = id >= pl.tail_items;
    if (it.prefix) id -= (int)pl.tail_items;
    const int tiles = it.prefix ? pl.prefix_tiles : pl.tail_tiles, parts = it.prefix ? pl.prefix_parts : pl.tail_parts;
    const int t = id / kXcds, unit = t / tiles * kXcds + id % kXcds, per = rows_of_sequence(g);
    int tile = t % tiles, keys, part = unit % parts;
    it.h = unit / parts % g.Hkv;
    if (it.prefix) {
        if (unit >= g.Hkv * parts) return false;
        int first, end;
        it.which = uniform(prefix_of_tile(g, rows, lane, tile, first, end, keys));
        if (it.which < 0) return false;
        it.row0 = first * per + tile * rows;
        it.row1 = min(it.row0 + rows, end * per);
        it.part = part;
    } else {
        if (unit >= g.batch * g.Hkv * parts) return false;
        it.which = unit / parts / g.Hkv;
        const int b = it.which;
        it.row0 = b * per + tile * rows;
        it.row1 = min(it.row0 + rows, (b + 1) * per);
        // up to the last key that a row of the tile sees
        const int fresh = fresh_of(g, b), lo = tile * rows, hi = it.row1 - b * per - 1;
        const int t_max = lo / g.n != hi / g.n ? g.n - 1 : hi % g.n;
        const int64_t seen = min((int64_t)g.pages.tail_len[b], (int64_t)g.pages.tail_len[b] - fresh + t_max + 1);
        keys = (int)min(max(seen, (int64_t)0), (int64_t)g.pages.table_width << g.pages.page_shift);
        it.part = (pl.prefix_parts > 0 ? pl.prefix_parts : 0) + part;
    }
    const int steps = (keys + step - 1) / step;
    it.begin = (int)((int64_t)part * steps / parts) * step;
    it.end = min(keys, (int)((int64_t)(part + 1) * steps / parts) * step);
    // (the same in all lanes, which the compiler cannot know of what was loaded)
    it.which = uniform(it.which);
    it.row0 = uniform(it.row0);
    it.row1 = uniform(it.row1);
    it.begin = uniform(it.begin);
    it.end = uniform(it.end);
    return true;
}

// Row number r of KV head h: its place in q and out; `limit`: the last tail token that it sees.  Rows of a prefix see
// everything, and so may those that are none (`live` false: padding, or behind the item's last), whose results go nowhere.
struct SharedRow {
    int b, hq, t, limit;
    bool live;
    __device__ __forceinline__ SharedRow(const SharedGeom &g, const SharedItem &it, int r) {
        const int per = rows_of_sequence(g), rr = min(r, it.row1 - 1);
        b = rr / per;
        const int at = rr - b * per, gi = at / g.n;
        hq = it.h * g.G + gi;
        t = at - gi * g.n;
        const int fresh = fresh_of(g, b);
        live = r < it.row1 && t < fresh;
        limit = !live || it.prefix ? INT_MAX : (int)max((int64_t)g.pages.tail_len[b] - fresh + t, (int64_t)-1);
    }
};

// Number of a row's partial result.
__device__ __forceinline__ int64_t partial_index(const SharedGeom &g, const SharedPlan &pl, int h, int part, int row) {
    return ((int64_t)h * (pl.prefix_parts + pl.tail_parts) + part) * g.batch * rows_of_sequence(g) + row;
}

// The keys of an item.
template <class T>
struct SharedKeys : KeyPlaces<T> {
    __device__ __forceinline__ SharedKeys(const SharedGeom &g, const SharedItem &it) {
        this->begin = it.begin;
        this->end = it.end;
        if (it.prefix)
            this->in_a_row((const T *)g.kp + it.which * g.ks[0] + it.h * g.ks[1], (const T *)g.vp + it.which * g.vs[0] + it.h * g.vs[1], g.ks[2],
                           g.vs[2]);
        else
            this->in_pages(g.pages, g.kt, g.vt, it.which, it.h);
    }
};

}  // namespace aha
