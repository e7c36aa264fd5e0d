// Where keys and values lie: in pages, or token by token.
#pragma once

#include "score_tile.h"

namespace aha {

// Where the key and value rows of a range of keys lie: `entry` is what there is to know of a key beforehand (its page), `at` the rows'
// offsets in elements from `k` and `v`; what is not there (beyond the end, in a hole) reads as zeros.
__device__ __attribute__((aligned(256))) const uint32_t kZeroRow[128] = {};
// A load from one of these: which of them a pointer is, the compiler cannot know, and its generic loads, which may be of LDS, are also counted with (and
// waited for like) LDS reads (fp32: 7 caches of up to 901 tokens 13.3 us, so 12.9).
template <class V>
__device__ __forceinline__ V load_global(const void *p) {
    return *(const __attribute__((address_space(1))) V *)(uintptr_t)p;
}
template <class T>
struct KeyPlaces {
    const T *k, *v;
    int64_t ks, vs;  // with a table: of a row in its page; without: of a token
    int64_t kp, vp;  // with a table: of a page
    const int32_t *table;
    int shift, pages, begin, end;
    __device__ __forceinline__ int entry(int key) const { return table ? table[min(key, end - 1) >> shift] : 0; }
    struct Row {
        const T *k, *v;
        bool there;
    };
    __device__ __forceinline__ Row at(int key, int page) const {
        Row r{(const T *)kZeroRow, (const T *)kZeroRow, key < end};
        if (table) {
            r.there = r.there && page >= 0 && page < pages;
            const int row = key & ((1 << shift) - 1);
            if (r.there) r.k = k + page * kp + row * ks, r.v = v + page * vp + row * vs;
        } else if (r.there) {
            r.k = k + key * ks, r.v = v + key * vs;
        }
        return r;
    }
    // keys of sequence b, KV head h, in pages; of one that lies token by token
    __device__ __forceinline__ void in_pages(const PageGeom &pg, const void *kt, const void *vt, int b, int h) {
        k = (const T *)kt + h * pg.ks[1];
        v = (const T *)vt + h * pg.vs[1];
        ks = pg.ks[2]; vs = pg.vs[2]; kp = pg.ks[0]; vp = pg.vs[0];
        table = pg.table + (int64_t)b * pg.table_width; shift = pg.page_shift; pages = pg.n_pages;
    }
    __device__ __forceinline__ void in_a_row(const T *k0, const T *v0, int64_t k_step, int64_t v_step) {
        k = k0; v = v0; ks = k_step; vs = v_step;
        kp = vp = 0; table = nullptr; shift = 0; pages = 0;
    }
};

}  // namespace aha
