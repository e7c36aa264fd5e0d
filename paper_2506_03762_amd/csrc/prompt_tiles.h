// Which rows a workgroup of the attention of packed prompts takes.
#pragma once

#include "key_places.h"

namespace aha {

// A tile: rows [row0, row1) of a prompt that begins at token lo, row1 - row0 at most `rows`; tokens counted from the tensors' start.
struct PromptTile {
    int lo, row0, row1, h, hq;
};

// prompt s: [lo, lo + n)
__device__ __forceinline__ int prompt_of(const PromptGeom &g, int s, int &lo) {
    lo = min(max(g.first[s], 0), g.tokens);
    return max(0, min(max(g.first[s + 1], 0), g.tokens) - lo);
}

// Number `k` of the prompts' tiles, the deepest first (a tile's keys are all tokens up to its last row), so that the last workgroups to
// start are short ones.  `t`: its number in its prompt.  The k-th is found by bisection over the depth, with the tiles of up to 256 prompts
// in registers, lane by lane; of more prompts the tiles are counted prompt by prompt.  All lanes of a wave call it and get the same.
__device__ __forceinline__ bool tile_of(const PromptGeom &g, int rows, int k, int lane, int &lo, int &n, int &t) {
    constexpr int U = 4;
    if (g.sequences <= 64 * U) {
        int tiles[U], begin[U], len[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int s = u * 64 + lane;
            tiles[u] = begin[u] = len[u] = 0;
            if (s < g.sequences) {
                len[u] = prompt_of(g, s, begin[u]);
                tiles[u] = (len[u] + rows - 1) / rows;
            }
        }
        auto deeper = [&](int depth) {  // tiles whose number in their prompt is at least `depth`
            int c = 0;
#pragma unroll
            for (int u = 0; u < U; ++u) c += max(0, tiles[u] - depth);
            return reduce_lanes<1, 64>(c, [](int a, int b) { return a + b; });
        };
        if (deeper(0) <= k) return false;
        int a = 0, b = (g.tokens + rows - 1) / rows;  // deeper(a) > k >= deeper(b)
        while (b - a > 1) {
            const int mid = (a + b) / 2;
            if (uniform(deeper(mid)) > k) a = mid; else b = mid;
        }
        t = a;
        int rank = k - uniform(deeper(b));  // among the prompts that have a tile of this number
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint64_t have = __builtin_amdgcn_ballot_w64(tiles[u] > t);
            const int count = __builtin_popcountll(have);
            if (rank < count) {
                const bool mine = tiles[u] > t && __builtin_amdgcn_mbcnt_hi((uint32_t)(have >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)have, 0)) == rank;
                const int at = __builtin_ctzll(__builtin_amdgcn_ballot_w64(mine));
                lo = __shfl(begin[u], at);
                n = __shfl(len[u], at);
                return true;
            }
            rank -= count;
        }
        return false;
    }
    for (int base = 0; base < g.sequences; base += 64) {
        int begin = 0, len = 0;
        if (base + lane < g.sequences) len = prompt_of(g, base + lane, begin);
        const int tiles = (len + rows - 1) / rows;
        int sum = tiles;  // over the lanes up to this one
#pragma unroll
        for (int s = 1; s < 64; s *= 2) {
            const int x = __shfl_up(sum, s);
            if (lane >= s) sum += x;
        }
        const uint64_t beyond = __builtin_amdgcn_ballot_w64(sum > k);
        if (beyond) {
            const int at = __builtin_ctzll(beyond);
            t = __shfl(tiles, at) - 1 - (k - __shfl(sum - tiles, at));
            lo = __shfl(begin, at);
            n = __shfl(len, at);
            return true;
        }
        k -= __shfl(sum, 63);
    }
    return false;
}

// Tile of workgroup `id`.  The query heads of a group, which read the same keys, get numbers that are congruent modulo the XCDs, whose
// workgroups share an L2.
__device__ __forceinline__ bool prompt_tile(const PromptGeom &g, int rows, int id, int lane, PromptTile &it) {
    const int x = id % kXcds, y = id / kXcds, unit = y / g.G * kXcds + x;
    int lo, n, t;
    it.h = unit % g.Hkv;
    it.hq = it.h * g.G + y % g.G;
    if (!tile_of(g, rows, unit / g.Hkv, lane, lo, n, t)) return false;
    it.lo = uniform(lo);
    it.row0 = uniform(lo + t * rows);
    it.row1 = uniform(lo + min(n, (t + 1) * rows));
    return true;
}

}  // namespace aha
