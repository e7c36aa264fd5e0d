// Eviction from a paged cache: of every (sequence, KV head) the tokens of the smallest scores go until `budget` are left, those that stay and lie
// behind the new length move into the places that became free.
//
// A token's rank is its key (class and score, order-preserving), its position (the highest goes first) and its place (the last goes first).
// One workgroup per (sequence, KV head) finds the rank of the last token to go, digit by digit, and lists the moves in order, with
// scores and positions; a second launch moves keys and values.
#include "aha_dev.h"
#include "aha_host.h"

namespace aha {

constexpr int kEvictThreads = 1024, kEvictWaves = kEvictThreads / 64;

// Ascending order of going: NaN, then scores, then protected tokens.
__device__ __forceinline__ uint32_t going_key(float f, bool safe) {
    const uint32_t u = __float_as_uint(f + 0.f);  // (-0 is 0)
    if (safe) return 0xffffffffu;
    if (f != f) return 0u;
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

struct EvictLds {
    int hist[256];
    int wave_count[2][kEvictWaves];
    int digit, rank;
};

// The value of rank `rank` (from 0) in ascending order of value(j), j of [0, n) with in(j); `rank` becomes the rank among those of
// this value.
template <class In, class Value>
__device__ __forceinline__ uint32_t value_of_rank(int n, int &rank, EvictLds &sm, In in, Value value) {
    const int tid = threadIdx.x;
    uint32_t found = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
        __syncthreads();
        if (tid < 256) sm.hist[tid] = 0;
        __syncthreads();
        for (int j = tid; j < n; j += kEvictThreads)
            if (in(j)) {
                const uint32_t x = value(j);
                if (shift == 24 || (x >> (shift + 8)) == (found >> (shift + 8))) atomicAdd(&sm.hist[(x >> shift) & 255], 1);
            }
        __syncthreads();
        if (tid < 64) {  // four digits per lane
            int c[4], sum = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) c[i] = sm.hist[tid * 4 + i], sum += c[i];
            int upto = sum;
#pragma unroll
            for (int s = 1; s < 64; s *= 2) {
                const int x = __shfl_up(upto, s);
                if (tid >= s) upto += x;
            }
            int below = upto - sum;
            if (rank >= below && rank < upto) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (rank >= below && rank < below + c[i]) sm.digit = tid * 4 + i, sm.rank = rank - below;
                    below += c[i];
                }
            }
        }
        __syncthreads();
        found |= (uint32_t)sm.digit << shift;
        rank = sm.rank;
    }
    return found;
}

__global__ __launch_bounds__(kEvictThreads) void evict_select_kernel(EvictGeom g, EvictPlan pl, int32_t *counts, int2 *moves) {
    __shared__ EvictLds sm;
    const int z = blockIdx.x, b = z / g.Hkv, h = z % g.Hkv, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t room = min((int64_t)g.pages.table_width << g.pages.page_shift, (int64_t)g.slots);
    const int len = max(0, (int)min((int64_t)g.pages.tail_len[b], room));
    const int64_t seen = (g.seen ? g.seen : g.pages.tail_len)[b];
    const int32_t *table = g.pages.table + (int64_t)b * g.pages.table_width;
    bool hole = false;
    for (int i = tid; i < (len + (1 << g.pages.page_shift) - 1) >> g.pages.page_shift; i += kEvictThreads)
        hole |= table[i] < 0 || table[i] >= g.pages.n_pages;
    const int keep = __syncthreads_or(hole) ? len : min(len, g.budget), go = len - keep;
    if (h == 0 && tid == 0) g.len_out[b] = keep;
    const float *scores = g.scores + b * g.ss[0] + h * g.ss[1];
    const int32_t *pos = g.pos ? g.pos + b * g.ps[0] + h * g.ps[1] : nullptr;
    float *scores_out = g.scores_out + b * g.so[0] + h * g.so[1];
    int32_t *pos_out = g.pos_out + b * g.po[0] + h * g.po[1];
    auto pos_of = [&](int j) { return pos ? pos[j] : j; };
    auto key_of = [&](int j) {
        const int p = pos_of(j);
        return going_key(scores[j], p >= seen - g.recent || p < g.sink);
    };
    int2 *mine = moves + (int64_t)z * pl.moves;
    int moved = 0;
    if (go > 0) {
        // the last token to go: key T, position P, place J
        auto high_first = [&](int j) { return ~((uint32_t)pos_of(j) ^ 0x80000000u); };
        auto last_first = [](int j) { return ~(uint32_t)j; };
        int rank = go - 1;
        const uint32_t T = value_of_rank(len, rank, sm, [](int) { return true; }, key_of);
        const uint32_t P = value_of_rank(len, rank, sm, [&](int j) { return key_of(j) == T; }, high_first);
        const uint32_t J = value_of_rank(len, rank, sm, [&](int j) { return key_of(j) == T && high_first(j) == P; }, last_first);
        auto goes = [&](int j) {
            const uint32_t k = key_of(j);
            if (k != T) return k < T;
            const uint32_t p = high_first(j);
            return p != P ? p < P : last_first(j) <= J;
        };
        // free places below `keep` and tokens that stay behind it, both in order
        int gaps = 0, movers = 0;
        for (int j0 = 0; j0 < len; j0 += kEvictThreads) {
            const int j = j0 + tid;
            const bool there = j < len, gone = there && goes(j), gap = gone && j < keep, mover = there && !gone && j >= keep;
            const uint64_t gm = __builtin_amdgcn_ballot_w64(gap), mm = __builtin_amdgcn_ballot_w64(mover);
            __syncthreads();
            if (lane == 0) sm.wave_count[0][wave] = __builtin_popcountll(gm), sm.wave_count[1][wave] = __builtin_popcountll(mm);
            __syncthreads();
            int before[2] = {gaps, movers};
            for (int w = 0; w < kEvictWaves; ++w) {
                const int c0 = sm.wave_count[0][w], c1 = sm.wave_count[1][w];
                if (w < wave) before[0] += c0, before[1] += c1;
                gaps += c0;
                movers += c1;
            }
            const uint64_t below = ((uint64_t)1 << lane) - 1;
            if (gap) mine[before[0] + __builtin_popcountll(gm & below)].x = j;
            if (mover) mine[before[1] + __builtin_popcountll(mm & below)].y = j;
        }
        moved = gaps;  // (as many as movers)
        __syncthreads();
    }
    if (tid == 0) counts[z] = moved;
    // every place that keeps its token, where the outputs are others than the inputs (moved ones are written behind the barrier)
    if (scores_out != scores)
        for (int j = tid; j < keep; j += kEvictThreads) scores_out[j] = scores[j];
    if (pos_out != pos)
        for (int j = tid; j < keep; j += kEvictThreads) pos_out[j] = pos_of(j);
    __syncthreads();
    for (int i = tid; i < moved; i += kEvictThreads) {
        const int2 mv = mine[i];
        scores_out[mv.x] = scores[mv.y];
        pos_out[mv.x] = pos_of(mv.y);
    }
}

// Keys and values of the moves: rows of `chunks` 16-byte chunks.
constexpr int kMoveRows = 16;  // of a workgroup
__global__ __launch_bounds__(256) void evict_move_kernel(EvictGeom g, EvictPlan pl, int chunks, const int32_t *counts, const int2 *moves) {
    const int z = blockIdx.y, b = z / g.Hkv, h = z % g.Hkv, count = counts[z], esize = g.dtype == AHA_BF16 ? 2 : 4;
    const int32_t *table = g.pages.table + (int64_t)b * g.pages.table_width;
    const int mask = (1 << g.pages.page_shift) - 1;
    for (int i = threadIdx.x; i < kMoveRows * chunks; i += 256) {
        const int at = blockIdx.x * kMoveRows + i / chunks, c = i % chunks;
        if (at >= count) return;
        const int2 mv = moves[(int64_t)z * pl.moves + at];
        const int to = table[mv.x >> g.pages.page_shift], from = table[mv.y >> g.pages.page_shift];
        auto move = [&](void *pool, const int64_t s[3]) {
            auto row = [&](int page, int j) { return (u32x4 *)((char *)pool + (page * s[0] + h * s[1] + (j & mask) * s[2]) * esize) + c; };
            *row(to, mv.x) = *row(from, mv.y);
        };
        move(g.kt, g.pages.ks);
        move(g.vt, g.pages.vs);
    }
}

hipError_t launch_paged_evict(const EvictGeom &g, const EvictPlan &pl, void *ws, hipStream_t st) {
    int32_t *counts = (int32_t *)ws;
    int2 *moves = (int2 *)((char *)ws + pl.off_moves);
    const int Z = g.batch * g.Hkv;
    hipLaunchKernelGGL(evict_select_kernel, dim3(Z), dim3(kEvictThreads), 0, st, g, pl, counts, moves);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || pl.moves == 0) return e;
    const int chunks = g.d * (g.dtype == AHA_BF16 ? 2 : 4) / 16;
    hipLaunchKernelGGL(evict_move_kernel, dim3((pl.moves + kMoveRows - 1) / kMoveRows, Z), dim3(256), 0, st, g, pl, chunks, counts, moves);
    return hipGetLastError();
}

}  // namespace aha
