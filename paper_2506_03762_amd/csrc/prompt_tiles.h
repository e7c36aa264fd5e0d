// Which rows a workgroup of the attention of packed prompts takes.
#pragma once

#include <algorithm>

#include "key_places.h"

namespace aha {

// The items of `pl`: a launch has fewer than 2^32 threads, so more than 2^23 workgroups of 256 take several (rows of a grid, whose width every workgroup has
// to read, cost all calls 0.2 us).
template <class Kernel>
static hipError_t launch_prompt_items(Kernel kernel, PromptGeom g, const PromptPlan &pl, size_t lds, hipStream_t st) {
    constexpr int64_t kMost = 1 << 23;
    for (int64_t i = 0; i < pl.items; i += kMost) {
        g.item0 = (int)i;
        hipLaunchKernelGGL(kernel, dim3((unsigned)std::min(kMost, pl.items - i)), dim3(256), lds, st, g);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// prompt s: [lo, lo + n)
__device__ __forceinline__ int prompt_of(const PromptGeom &g, int s, int &lo) {
    lo = min(max(g.first[s], 0), g.tokens);
    return max(0, min(max(g.first[s + 1], 0), g.tokens) - lo);
}

// Number `k` of the prompts' tiles, of which a prompt of n tokens has tiles_of(n): prompt by prompt, so that workgroups that run at the same time
// read the same keys from their L2, the longest first, and of a prompt the deepest first (a tile's keys are all tokens up to its last
// row), so that the last workgroups to start are short ones (the deepest of all prompts first: 24 prompts of up to 1500 tokens, 8 x 4 heads, 1.07 us
// for the products of 32 keys and 256 rows instead of 0.85).  More than 64 prompts are taken in their own order, 256 to a look (1000
// prompts of 64 tokens, 8 heads of 128 over 2, 108 us, with 64 to a look 148).
// `lo`, `n`: its prompt, `t`: its number there.  All lanes of a wave call it and get the same.
template <class TilesOf>
__device__ __forceinline__ bool tile_of(const PromptGeom &g, int k, int lane, int &lo, int &n, int &t, TilesOf tiles_of) {
    if (g.sequences <= 64) {  // (one to a lane)
        int begin = 0, len = 0, before = 0;  // tiles of the prompts before the lane's
        if (lane < g.sequences) len = prompt_of(g, lane, begin);
        const int tiles = tiles_of(len);
        const uint32_t order = (uint32_t)tiles * 64 + 63 - lane;  // (no two the same; fewer than 2^26 tiles)
        for (int s0 = 0; s0 < g.sequences; s0 += 8)
#pragma unroll
            for (int s = 0; s < 8; ++s) {  // (lanes without a prompt add nothing)
                const uint32_t other = __builtin_amdgcn_readlane(order, s0 + s);
                before += other > order ? other / 64 : 0;
            }
        const uint64_t mine = __builtin_amdgcn_ballot_w64(k >= before && k < before + tiles);
        if (mine == 0) return false;
        const int at = __builtin_ctzll(mine);
        lo = __builtin_amdgcn_readlane(begin, at);
        n = __builtin_amdgcn_readlane(len, at);
        t = __builtin_amdgcn_readlane(before + tiles, at) - 1 - k;
        return true;
    }
    for (int base = 0; base < g.sequences; base += 256) {  // four consecutive ones to a lane
        int begin[5], tiles[4], own = 0;
#pragma unroll
        for (int i = 0; i < 5; ++i) begin[i] = min(max(g.first[min(base + 4 * lane + i, g.sequences)], 0), g.tokens);
#pragma unroll
        for (int i = 0; i < 4; ++i) tiles[i] = tiles_of(max(0, begin[i + 1] - begin[i])), own += tiles[i];
        int sum = own;  // over the lanes up to this one
#pragma unroll
        for (int s = 1; s < 64; s *= 2) {
            const int x = __shfl_up(sum, s);
            if (lane >= s) sum += x;
        }
        const uint64_t beyond = __builtin_amdgcn_ballot_w64(sum > k);
        if (beyond) {
            const int at = __builtin_ctzll(beyond);
            k -= __builtin_amdgcn_readlane(sum - own, at);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int here = __builtin_amdgcn_readlane(tiles[i], at);
                if (k < here) {
                    lo = __builtin_amdgcn_readlane(begin[i], at);
                    n = __builtin_amdgcn_readlane(begin[i + 1], at) - lo;
                    t = here - 1 - k;
                    return true;
                }
                k -= here;
            }
        }
        k -= __builtin_amdgcn_readlane(sum, 63);
    }
    return false;
}

// Tiles of `rows` rows of one query head: rows [row0, row1) of a prompt that begins at token lo, counted from the tensors' start.  The query heads of
// a group, which read the same keys, get numbers that are congruent modulo the XCDs, whose workgroups share an L2.
struct PromptTile {
    int lo, row0, row1, h, hq;
};
__device__ __forceinline__ bool prompt_tile(const PromptGeom &g, int rows, int id, int lane, PromptTile &it) {
    const int x = id % kXcds, y = id / kXcds, unit = y / g.G * kXcds + x;
    int lo, n, t;
    it.h = unit % g.Hkv;
    it.hq = it.h * g.G + y % g.G;
    if (!tile_of(g, unit / g.Hkv, lane, lo, n, t, [&](int len) { return (len + rows - 1) / rows; })) return false;
    it.lo = uniform(lo);
    it.row0 = uniform(lo + t * rows);
    it.row1 = uniform(lo + min(n, (t + 1) * rows));
    return true;
}

// Tiles of kUnits units, a unit being 64 rows of one of the query heads of a KV head: a prompt's units are its blocks of 64 rows times the heads of the
// group, heads first, so that the units of a tile see nearly the same keys (4 heads: the same ones.  24 prompts of up to 1500 tokens, 8 x 4
// heads 343 us with 256 rows of one head to a tile).
struct PromptUnits {
    int lo, n, h, first, end;  // the prompt, its tokens, the KV head, the first unit, keys of the tile
};
constexpr int kUnits = 4;
template <int ROWS>
__device__ __forceinline__ bool prompt_units(const PromptGeom &g, int id, int lane, PromptUnits &it) {
    int lo, n, t;
    it.h = id % g.Hkv;
    auto units = [&](int len) { return (len + ROWS - 1) / ROWS * g.G; };
    if (!tile_of(g, id / g.Hkv, lane, lo, n, t, [&](int len) { return (units(len) + kUnits - 1) / kUnits; })) return false;
    it.lo = uniform(lo);
    it.n = uniform(n);
    it.first = uniform(t * kUnits);
    it.end = min(it.n, (min(it.first + kUnits, units(it.n)) - 1) / g.G * ROWS + ROWS);
    return true;
}

}  // namespace aha
