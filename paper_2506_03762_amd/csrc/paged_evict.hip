// Eviction from a paged cache: of every (sequence, KV head) the tokens of the smallest scores go until `budget` are left, those that stay and lie
// behind the new length move into the places that became free.
//
// A token's rank is its key (class and score, order-preserving), its position (the highest goes first) and its place (the last goes first).
// One workgroup per (sequence, KV head) finds the rank of the last token to go, lists the moves in order and moves scores and positions;
// it moves the keys and values too where there can only be a few, else a second launch does.
//
// The selection is bound by what one CU does for a row of scores: every key is read from memory once and from LDS three times (histogram, counts, lists), so
// 32768 tokens of 8 heads take 22 us, 2049 of 64 x 8 heads, of which one goes, 8.8.  More CUs to a row would need two more launches.  Where the keys do not
// fit, they are formed again from scores and positions in each of the four sweeps: 131072 tokens of 8 heads 118 us with the moves (digit by digit of the last
// one's rank, twelve sweeps, 447).  The moves are bound by memory: 8 prompts of up to 16384 tokens to 2048, 112 MB in 24 us, 4.7 TB/s.
#include <limits.h>

#include <algorithm>
#include <type_traits>

#include "aha_dev.h"
#include "aha_host.h"

namespace aha {

// Ascending order of going: NaN, then scores, then protected tokens.
constexpr uint32_t kSafe = 0xffffffffu;
__device__ __forceinline__ uint32_t going_key(float f, bool safe) {
    const uint32_t u = __float_as_uint(f + 0.f);  // (-0 is 0)
    const uint32_t key = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
    return safe ? kSafe : f != f ? 0u : key;
}

// The rank of a token; small ones go.
struct Rank {
    uint64_t what;   // key, then the position: the highest first
    uint32_t place;  // the last first
    __device__ __forceinline__ bool operator<(const Rank &o) const { return what != o.what ? what < o.what : place < o.place; }
};
__device__ __forceinline__ uint64_t rank_what(uint32_t key, int pos) { return (uint64_t)key << 32 | (uint32_t)~((uint32_t)pos ^ 0x80000000u); }

template <int WAVES>
struct EvictLds {
    // four bins to a thread; tokens that are ranked by comparing them all, where last_to_go() takes longer (rows of 900, 4000, 32000 tokens: 300 alike
    // 28, 32, 43 us ranked, 22, 32, 68 by it; 180 18, 26, 36)
    static constexpr int kBins = WAVES * 256, kCandidates = 160 + 28 * WAVES;
    union {
        alignas(16) int hist[kBins];
        Rank candidates[kCandidates];
    };
    uint32_t all_low, all_above, from, to;
    int all_free;
    int count[2][WAVES], gaps[WAVES], movers[WAVES];
    Rank best[WAVES], last;
    int digit, rank, in_bin, n_candidates;
};

__device__ __forceinline__ int wave_add(int x) {
    return reduce_lanes<1, 64>(x, [](int a, int b) { return a + b; });
}
// Sum over the lanes up to this one.
__device__ __forceinline__ int wave_prefix(int x, int lane) {
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
        const int y = __shfl_up(x, s);
        if (lane >= s) x += y;
    }
    return x;
}

// What a workgroup reads of its tokens.
struct EvictRows {
    const float *scores;
    const int32_t *pos;
    int safe_from, sink;  // positions that are protected: from the one on, before the other
    __device__ __forceinline__ int pos_of(int j) const { return pos ? pos[j] : j; }
    __device__ __forceinline__ bool safe(int p) const { return p >= safe_from || p < sink; }
    __device__ __forceinline__ uint32_t key_of(float score, int p) const { return going_key(score, safe(p)); }
    __device__ __forceinline__ uint32_t key_at(int j) const { return key_of(scores[j], pos_of(j)); }
};

// Keys and values of moves, in rows of 16-byte chunks.
__device__ __forceinline__ void move_rows(const EvictGeom &g, const int32_t *table, int h, const int2 *moves, int count, int tid, int threads) {
    const int esize = g.dtype == AHA_BF16 ? 2 : 4, chunks = g.d * esize / 16, mask = (1 << g.pages.page_shift) - 1;
    auto row = [&](void *pool, const int64_t s[3], int j, int chunk) {
        return (u32x4 *)((char *)pool + (table[j >> g.pages.page_shift] * s[0] + h * s[1] + (j & mask) * s[2]) * esize) + chunk;
    };
    constexpr int U = 4;  // rows' chunks in flight
    for (int i0 = tid; i0 < count * chunks; i0 += U * threads) {
        u32x4 k[U], v[U];
        int2 mv[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * threads;
            if (i < count * chunks) mv[u] = moves[i / chunks];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * threads;
            if (i < count * chunks) k[u] = *row(g.kt, g.pages.ks, mv[u].y, i % chunks), v[u] = *row(g.vt, g.pages.vs, mv[u].y, i % chunks);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * threads;
            if (i < count * chunks) *row(g.kt, g.pages.ks, mv[u].x, i % chunks) = k[u], *row(g.vt, g.pages.vs, mv[u].x, i % chunks) = v[u];
        }
    }
}

__device__ __forceinline__ int mask_number(uint64_t m, int from) {  // `from` plus the lanes below this one whose bit is set
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, from));
}
// What a workgroup does: `len` tokens, of which `keep` stay.
struct Eviction {
    EvictRows rows;
    float *scores_out;
    int32_t *pos_out;
    int2 *moves;
    int len, keep;
    // token `from` goes to place `to`
    __device__ __forceinline__ void move(int i, int to, int from) const {
        moves[i] = make_int2(to, from);
        scores_out[to] = rows.scores[from];
        pos_out[to] = rows.pos_of(from);
    }
    // every place that keeps its token, where the outputs are others than the inputs (places that get another one are written behind a
    // barrier)
    __device__ __forceinline__ void copy(int tid, int threads) const {
        const bool s = scores_out != rows.scores, p = pos_out != rows.pos;
        if (!s && !p) return;
        for (int j = tid; j < keep; j += 4 * threads) {
            float x[4];
            int y[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) x[u] = rows.scores[min(j + u * threads, keep - 1)], y[u] = rows.pos_of(min(j + u * threads, keep - 1));
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (j + u * threads < keep) {
                    if (s) scores_out[j + u * threads] = x[u];
                    if (p) pos_out[j + u * threads] = y[u];
                }
        }
    }
};

// A histogram, linear over a range of keys: the bin of the last one to go, whose keys are then ranked against each other.
template <int WAVES>
struct EvictBins {
    uint32_t low, high, slope;
    // a little less than kBins 2^32 / (range + 1), which 64-bit division would take all waves 1.5 us for; 0: a bin for every key
    __device__ __forceinline__ EvictBins(uint32_t low_, uint32_t high_) : low(low_), high(high_) {
        constexpr int kBins = EvictLds<WAVES>::kBins;
        const uint32_t range = high - low;
        slope = range < kBins ? 0u : (uint32_t)(kBins * 0x1p32f * (1.f - 0x1p-20f) * __builtin_amdgcn_rcpf((float)range + 1.f));
    }
    __device__ __forceinline__ int bin_of(uint32_t k) const { return (int)(slope ? __umulhi(k - low, slope) : k - low); }
    __device__ __forceinline__ uint64_t first_of(int bin) const {
        return low + (slope ? (((uint64_t)bin << 32) + slope - 1) / slope : (uint64_t)bin);
    }
    // The bin that the last of `go` lies in: its keys are those from sm.from up to sm.to (smaller ones go, larger ones stay), sm.in_bin of them, of which
    // number sm.rank from the smallest on is the last one.  All threads call it, between barriers of its own.
    __device__ __forceinline__ void find(EvictLds<WAVES> &sm, int go, int tid) const {
        const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        __syncthreads();
        const u32x4 c = *(const u32x4 *)&sm.hist[4 * tid];
        const int sum = (int)((c[0] + c[1]) + (c[2] + c[3]));
        int below = wave_prefix(sum, lane);
        if (lane == 63) sm.count[1][wave] = below;
        __syncthreads();
        below -= sum;
        for (int w = 0; w < wave; ++w) below += sm.count[1][w];
        if (go > below && go <= below + sum) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (go > below && go <= below + (int)c[i]) sm.digit = tid * 4 + i, sm.rank = go - 1 - below, sm.in_bin = (int)c[i];
                below += c[i];
            }
            sm.from = (uint32_t)first_of(sm.digit);
            sm.to = (uint32_t)min(first_of(sm.digit + 1) - 1, (uint64_t)high);
        }
        __syncthreads();
    }
};
// The candidates, noted by all waves, ranked: sm.last is the last one to go, and what the waves have counted (sm.gaps, sm.movers; `per_wave` tokens to a wave)
// is made complete.  Begins and ends with a barrier.
template <int WAVES>
__device__ __forceinline__ void rank_candidates(EvictLds<WAVES> &sm, int keep, int per_wave, int tid) {
    const int in_bin = sm.in_bin, want = sm.rank;
    __syncthreads();
    for (int i = tid; i < in_bin; i += WAVES * 64) {
        const Rank r = sm.candidates[i];
        int smaller = 0;
#pragma unroll 8
        for (int o = 0; o < in_bin; ++o) smaller += sm.candidates[o] < r;
        if (smaller == want) sm.last = r;
        // (what the rank says, too: the first want + 1 of them go)
        const int j = (int)~r.place, w = j / per_wave;
        if (smaller <= want && j < keep) atomicAdd(&sm.gaps[w], 1);
        if (smaller > want && j >= keep) atomicAdd(&sm.movers[w], 1);
    }
    __syncthreads();
}

// The last one to go of many alike: number `want` of the `left` tokens whose keys lie in [k0, k1].  Histograms of these keys, then of the positions of an only
// key, then of the places of an only position, until so few are left that they are ranked (63 rows of 1891 scores of 0 18 us, different scores 16; digit by
// digit of key, position and place 36).
template <int WAVES>
__device__ __forceinline__ Rank last_to_go(const EvictRows &rows, int len, int want, int left, uint32_t k0, uint32_t k1, EvictLds<WAVES> &sm, int tid) {
    constexpr int THREADS = WAVES * 64, U = 8;
    uint32_t p0 = 0, p1 = ~0u, j0 = ~(uint32_t)(len - 1), j1 = ~0u;  // what is known of its position and place
    // work(key, position's rank, place's rank) for the tokens left
    auto sweep = [&](auto work) {
        for (int first = tid; first < len; first += U * THREADS) {
            float score[U];
            int pos[U];
#pragma unroll
            for (int u = 0; u < U; ++u) score[u] = rows.scores[min(first + u * THREADS, len - 1)], pos[u] = rows.pos_of(min(first + u * THREADS, len - 1));
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint64_t what = rank_what(rows.key_of(score[u], pos[u]), pos[u]);
                const uint32_t k = (uint32_t)(what >> 32), p = (uint32_t)what, place = ~(uint32_t)(first + u * THREADS);
                if (first + u * THREADS < len && k >= k0 && k <= k1 && p >= p0 && p <= p1 && place >= j0 && place <= j1) work(k, p, place);
            }
        }
    };
    auto narrow = [&](uint32_t &from, uint32_t &to, auto value) {
        const EvictBins<WAVES> bins(from, to);
        __syncthreads();
        *(u32x4 *)&sm.hist[4 * tid] = u32x4{0, 0, 0, 0};
        __syncthreads();
        sweep([&](uint32_t k, uint32_t p, uint32_t place) { atomicAdd(&sm.hist[bins.bin_of(value(k, p, place))], 1); });
        bins.find(sm, want + 1, tid);
        from = sm.from;
        to = sm.to;
        want = sm.rank;
        left = sm.in_bin;
    };
    while (left > sm.kCandidates && k0 < k1) narrow(k0, k1, [](uint32_t k, uint32_t, uint32_t) { return k; });
    if (left > sm.kCandidates) {  // the range of their positions
        uint32_t low = ~0u, high = 0;
        sweep([&](uint32_t, uint32_t p, uint32_t) { low = min(low, p), high = max(high, p); });
        low = reduce_lanes<1, 64>(low, OpMinU{});
        high = reduce_lanes<1, 64>(high, OpMaxU{});
        __syncthreads();
        if (tid == 0) sm.all_low = ~0u, sm.all_above = 0;
        __syncthreads();
        if ((tid & 63) == 0) atomicMin(&sm.all_low, low), atomicMax(&sm.all_above, high);
        __syncthreads();
        p0 = sm.all_low;
        p1 = sm.all_above;
    }
    while (left > sm.kCandidates && p0 < p1) narrow(p0, p1, [](uint32_t, uint32_t p, uint32_t) { return p; });
    while (left > sm.kCandidates) narrow(j0, j1, [](uint32_t, uint32_t, uint32_t place) { return place; });
    __syncthreads();
    if (tid == 0) sm.n_candidates = 0;
    __syncthreads();
    sweep([&](uint32_t k, uint32_t p, uint32_t place) { sm.candidates[atomicAdd(&sm.n_candidates, 1)] = Rank{(uint64_t)k << 32 | p, place}; });
    __syncthreads();
    for (int i = tid; i < left; i += THREADS) {
        const Rank r = sm.candidates[i];
        int smaller = 0;
#pragma unroll 8
        for (int o = 0; o < left; ++o) smaller += sm.candidates[o] < r;
        if (smaller == want) sm.last = r;
    }
    __syncthreads();
    return sm.last;
}

// The tokens' keys in LDS, `steps` steps of 64 tokens of a wave, one lane each, which alone reads them.  Returns the number of moves.
// (`holes`: all threads call it; whether the sequence has one)
template <int WAVES, class Holes>
__device__ __forceinline__ int evict_in_lds(Eviction &e, EvictLds<WAVES> &sm, uint32_t *keys, uint16_t *gap_places, int tid, Holes holes) {
    constexpr int THREADS = WAVES * 64, U = WAVES == 16 ? 16 : 4;
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), len = e.len;
    const int per_wave = (len + THREADS - 1) / THREADS * 64, first = wave * per_wave, steps = min(per_wave, max(0, len - first) + 63) / 64;
    const int base = first + lane;
    const EvictRows &rows = e.rows;
    uint32_t *key = keys + base;
    if (tid == 0) sm.all_low = kSafe, sm.all_above = 0, sm.all_free = 0, sm.n_candidates = 0;
    // the range of the keys that may go, and their number
    uint32_t low = kSafe, above = 0;
    int free_keys = 0;
    auto count = [&](uint32_t k) {
        low = min(low, k);
        above = max(above, k + 1);  // (0 of protected ones)
        free_keys += __builtin_popcountll(__builtin_amdgcn_ballot_w64(k != kSafe));
    };
    // U steps' scores and positions are requested before any is used; WHOLE: all U of them, and no place behind the last token (with 32 steps an
    // instruction per step takes the 16 waves 0.24 us)
    auto batch = [&](auto whole, int t0) {
        constexpr bool WHOLE = decltype(whole)::value;
        uint32_t score[U], top = 0;
        int pos[U];
        const float *scores = rows.scores + base + t0 * 64;
        const int32_t *given = rows.pos + base + t0 * 64;
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (WHOLE || t0 + u < steps) score[u] = __float_as_uint(WHOLE ? scores[u * 64] : rows.scores[min(base + (t0 + u) * 64, len - 1)]);
        if (rows.pos) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (WHOLE || t0 + u < steps) pos[u] = WHOLE ? given[u * 64] : rows.pos[min(base + (t0 + u) * 64, len - 1)];
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (WHOLE || t0 + u < steps) top = max(top, score[u]);
        // no protected token, no negative score, -0 or NaN
        const int j0 = first + t0 * 64, j1 = j0 + U * 64;
        if (WHOLE && !rows.pos && j0 >= rows.sink && j1 <= rows.safe_from && __builtin_amdgcn_ballot_w64(top > 0x7f800000u) == 0) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint32_t k = score[u] | 0x80000000u;
                low = min(low, k);
                key[(t0 + u) * 64] = k;
            }
            above = max(above, (top | 0x80000000u) + 1);
            free_keys += U * 64;
            return;
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (WHOLE || t0 + u < steps) {
                const int j = base + (t0 + u) * 64;
                uint32_t k = rows.key_of(__uint_as_float(score[u]), rows.pos ? pos[u] : j);
                if (!WHOLE && j >= len) k = kSafe;  // (counts as a protected one; `rank_of` is asked of tokens alone)
                key[(t0 + u) * 64] = k;
                count(k);
            }
    };
    for (int t0 = 0; t0 < steps; t0 += U) {
        if (t0 + U <= steps && first + (t0 + U) * 64 <= len) batch(std::true_type{}, t0);
        else batch(std::false_type{}, t0);
    }
    if (holes()) {  // (behind a barrier)
        e.keep = len;
        return 0;
    }
    const int keep = e.keep, go = len - keep;
    auto rank_of = [&](int t, uint32_t k) { return Rank{rank_what(k, rows.pos_of(base + t * 64)), ~(uint32_t)(base + t * 64)}; };
    auto of_all = [&] {
        low = reduce_lanes<1, 64>(low, OpMinU{});
        above = reduce_lanes<1, 64>(above, OpMaxU{});
        if (lane == 0) atomicMin(&sm.all_low, low), atomicMax(&sm.all_above, above), atomicAdd(&sm.all_free, free_keys);
        __syncthreads();
        low = sm.all_low;
        above = sm.all_above;
        free_keys = sm.all_free;
    };
    if (go > 1)
        *(u32x4 *)&sm.hist[4 * tid] = u32x4{0, 0, 0, 0};
    of_all();
    const bool turned = go > free_keys;
    const int unprotected = free_keys;
    if (turned) {  // all that may go do, and protected ones by their position: other keys of the same order, positions in turns
        __syncthreads();
        if (tid == 0) sm.all_low = kSafe, sm.all_above = 0, sm.all_free = 0;
#pragma unroll 8
        for (int t = 0; t < steps; ++t)
            if (base + t * 64 < len)
                key[t * 64] = key[t * 64] == kSafe ? min(max((uint32_t)rank_what(0, rows.pos_of(base + t * 64)), 1u), kSafe - 1) : 0u;
        low = kSafe, above = 0, free_keys = 0;
        for (int t = 0; t < steps; ++t) count(key[t * 64]);
        __syncthreads();
        of_all();
    }
    Rank last;
    if (go == 1) {  // the smallest
        Rank best{~(uint64_t)0, ~0u};
        bool any = false;
        for (int t = 0; t < steps; ++t)
            if (key[t * 64] == low && base + t * 64 < len) {
                const Rank r = rank_of(t, low);
                if (r < best) best = r;
                any = true;
            }
        if (__builtin_amdgcn_ballot_w64(any)) {
#pragma unroll
            for (int s = 32; s > 0; s /= 2) {
                const Rank r{__shfl_xor((unsigned long long)best.what, s), (uint32_t)__shfl_xor((int)best.place, s)};
                if (r < best) best = r;
            }
        }
        if (lane == 0) sm.best[wave] = best;
        __syncthreads();
        last = sm.best[0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w)
            if (sm.best[w] < last) last = sm.best[w];
        const int gone = (int)~last.place;
        if (gone >= keep) return 0;  // (the last token itself)
        if (tid == 0) e.move(0, gone, keep);
        return 1;
    }
    // free places below `keep` and tokens that stay behind it are listed, both in order: steps with places below `keep`, the first step with others
    const int front_steps = min(steps, max(0, keep - first + 63) / 64), back = min(steps, max(0, keep - first) / 64);
    int gaps = 0, movers = 0;
    bool found = false;
    {
        const EvictBins<WAVES> bins(low, above - 1);
#pragma unroll 4
        for (int t = 0; t < steps; ++t) {
            const uint32_t k = key[t * 64];
            if (k != kSafe) atomicAdd(&sm.hist[bins.bin_of(k)], 1);
        }
        bins.find(sm, go, tid);
        const uint32_t from = sm.from, to = sm.to;
        if (sm.in_bin <= sm.kCandidates) {
            found = true;
            auto note = [&](int t) {
                const uint32_t k = key[t * 64];
                if (k >= from && k <= to) sm.candidates[atomicAdd(&sm.n_candidates, 1)] = rank_of(t, k);
                return k;
            };
            int t = 0;
#pragma unroll 8
            for (; t < back; ++t) gaps += __builtin_popcountll(__builtin_amdgcn_ballot_w64(note(t) < from));
            if (t < front_steps) {  // (the step that `keep` lies in)
                const uint32_t k = note(t);
                const int j = base + t * 64;
                gaps += __builtin_popcountll(__builtin_amdgcn_ballot_w64(k < from && j < keep));
                movers += __builtin_popcountll(__builtin_amdgcn_ballot_w64(k > to && j >= keep && j < len));
                ++t;
            }
#pragma unroll 8
            for (; t < steps; ++t) {
                uint64_t stays = __builtin_amdgcn_ballot_w64(note(t) > to);
                if (first + t * 64 + 64 > len) stays &= ((uint64_t)1 << (len - first - t * 64)) - 1;
                movers += __builtin_popcountll(stays);
            }
            if (lane == 0) sm.gaps[wave] = gaps, sm.movers[wave] = movers;
            rank_candidates(sm, keep, per_wave, tid);
            last = sm.last;
        }
    }
    // what goes now has keys up to `last_key`, what stays larger ones
    uint32_t last_key;
    if (found) {
        last_key = (uint32_t)(last.what >> 32);
        for (int i = tid; i < sm.in_bin; i += THREADS) {
            const Rank r = sm.candidates[i];
            if ((uint32_t)(r.what >> 32) == last_key && last < r) keys[~r.place] = kSafe;
        }
    } else {
        last = turned ? last_to_go(rows, len, go - 1 - unprotected, len - unprotected, kSafe, kSafe, sm, tid)
                      : last_to_go(rows, len, sm.rank, sm.in_bin, sm.from, sm.to, sm, tid);
        last_key = 0;
#pragma unroll 8
        for (int t = 0; t < steps; ++t)
            if (base + t * 64 < len) key[t * 64] = last < rank_of(t, rows.key_at(base + t * 64)) ? kSafe : 0u;
        for (int t = 0; t < front_steps; ++t) gaps += __builtin_popcountll(__builtin_amdgcn_ballot_w64(key[t * 64] == 0 && base + t * 64 < keep));
        for (int t = back; t < steps; ++t)
            movers += __builtin_popcountll(__builtin_amdgcn_ballot_w64(key[t * 64] != 0 && (uint32_t)(base + t * 64 - keep) < (uint32_t)go));
        if (lane == 0) sm.gaps[wave] = gaps, sm.movers[wave] = movers;
    }
    __syncthreads();
    gaps = movers = 0;
    int moved = 0;
    for (int w = 0; w < WAVES; ++w) {
        moved += sm.gaps[w];  // (as many as movers)
        if (w < wave) gaps += sm.gaps[w], movers += sm.movers[w];
    }
    gaps = __builtin_amdgcn_readfirstlane(gaps);
    movers = __builtin_amdgcn_readfirstlane(movers);
    uint16_t *mover_places = gap_places + moved;
#pragma unroll 8
    for (int t = 0; t < front_steps; ++t) {
        const bool gap = key[t * 64] <= last_key && base + t * 64 < keep;
        const uint64_t m = __builtin_amdgcn_ballot_w64(gap);
        if (gap) gap_places[mask_number(m, gaps)] = (uint16_t)(base + t * 64);
        gaps += __builtin_popcountll(m);
    }
#pragma unroll 8
    for (int t = back; t < steps; ++t) {
        const bool mover = key[t * 64] > last_key && (uint32_t)(base + t * 64 - keep) < (uint32_t)go;
        const uint64_t m = __builtin_amdgcn_ballot_w64(mover);
        if (mover) mover_places[mask_number(m, movers)] = (uint16_t)(base + t * 64);
        movers += __builtin_popcountll(m);
    }
    __syncthreads();
    for (int i = tid; i < moved; i += THREADS) e.move(i, gap_places[i], mover_places[i]);
    return moved;
}

// More tokens than that: their keys are formed again whenever they are needed.  `holes` as above; the moves' lists are `e.moves` themselves.
template <int WAVES, class Holes>
__device__ __forceinline__ int evict_from_memory(Eviction &e, EvictLds<WAVES> &sm, int tid, Holes holes) {
    constexpr int THREADS = WAVES * 64, U = 8;
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), len = e.len;
    const int per_wave = (len + THREADS * U - 1) / (THREADS * U) * 64 * U, first = wave * per_wave, end = min(len, first + per_wave);
    const EvictRows &rows = e.rows;
    // work(j, key) for the wave's tokens, one per lane (behind the last token a protected one's); U steps' scores and positions are in flight
    auto sweep = [&](auto work) {
        for (int j0 = first + lane; j0 - lane < end; j0 += U * 64) {
            float score[U];
            int pos[U];
#pragma unroll
            for (int u = 0; u < U; ++u) score[u] = rows.scores[min(j0 + u * 64, len - 1)], pos[u] = rows.pos_of(min(j0 + u * 64, len - 1));
#pragma unroll
            for (int u = 0; u < U; ++u) work(j0 + u * 64, j0 + u * 64 < end ? rows.key_of(score[u], pos[u]) : kSafe, pos[u]);
        }
    };
    if (tid == 0) sm.all_low = kSafe, sm.all_above = 0, sm.all_free = 0, sm.n_candidates = 0;
    *(u32x4 *)&sm.hist[4 * tid] = u32x4{0, 0, 0, 0};
    uint32_t low = kSafe, above = 0;
    int free_keys = 0;
    sweep([&](int, uint32_t k, int) {
        low = min(low, k);
        above = max(above, k + 1);  // (0 of protected ones)
        free_keys += __builtin_popcountll(__builtin_amdgcn_ballot_w64(k != kSafe));
    });
    if (holes()) {  // (behind a barrier)
        e.keep = len;
        return 0;
    }
    const int keep = e.keep, go = len - keep;
    low = reduce_lanes<1, 64>(low, OpMinU{});
    above = reduce_lanes<1, 64>(above, OpMaxU{});
    if (lane == 0) atomicMin(&sm.all_low, low), atomicMax(&sm.all_above, above), atomicAdd(&sm.all_free, free_keys);
    __syncthreads();
    Rank last;
    int gaps = 0, movers = 0;
    bool found = false;
    if (go <= sm.all_free) {
        const EvictBins<WAVES> bins(sm.all_low, sm.all_above - 1);
        sweep([&](int, uint32_t k, int) {
            if (k != kSafe) atomicAdd(&sm.hist[bins.bin_of(k)], 1);
        });
        bins.find(sm, go, tid);
        const uint32_t from = sm.from, to = sm.to;
        if (sm.in_bin <= sm.kCandidates) {
            found = true;
            sweep([&](int j, uint32_t k, int p) {
                if (k >= from && k <= to) sm.candidates[atomicAdd(&sm.n_candidates, 1)] = Rank{rank_what(k, p), ~(uint32_t)j};
                gaps += __builtin_popcountll(__builtin_amdgcn_ballot_w64(k < from && j < keep));
                movers += __builtin_popcountll(__builtin_amdgcn_ballot_w64(k > to && j >= keep && j < end));
            });
            if (lane == 0) sm.gaps[wave] = gaps, sm.movers[wave] = movers;
            rank_candidates(sm, keep, per_wave, tid);
            last = sm.last;
        }
    }
    auto goes = [&](int j, uint32_t k, int p) { return !(last < Rank{rank_what(k, p), ~(uint32_t)j}); };
    if (!found) {  // protected tokens go, or too many keys are alike
        last = go > sm.all_free ? last_to_go(rows, len, go - 1 - sm.all_free, len - sm.all_free, kSafe, kSafe, sm, tid)
                                : last_to_go(rows, len, sm.rank, sm.in_bin, sm.from, sm.to, sm, tid);
        sweep([&](int j, uint32_t k, int p) {
            const bool out = goes(j, k, p);
            gaps += __builtin_popcountll(__builtin_amdgcn_ballot_w64(out && j < min(keep, end)));
            movers += __builtin_popcountll(__builtin_amdgcn_ballot_w64(!out && j >= keep && j < end));
        });
        if (lane == 0) sm.gaps[wave] = gaps, sm.movers[wave] = movers;
        __syncthreads();
    }
    gaps = movers = 0;
    int moved = 0;
    for (int w = 0; w < WAVES; ++w) {
        moved += sm.gaps[w];  // (as many as movers)
        if (w < wave) gaps += sm.gaps[w], movers += sm.movers[w];
    }
    sweep([&](int j, uint32_t k, int p) {
        const bool out = goes(j, k, p), gap = out && j < min(keep, end), mover = !out && j >= keep && j < end;
        const uint64_t gm = __builtin_amdgcn_ballot_w64(gap), mm = __builtin_amdgcn_ballot_w64(mover);
        if (gap) e.moves[mask_number(gm, gaps)].x = j;
        if (mover) e.moves[mask_number(mm, movers)].y = j;
        gaps += __builtin_popcountll(gm);
        movers += __builtin_popcountll(mm);
    });
    __syncthreads();
    for (int i = tid; i < moved; i += THREADS) {
        const int2 mv = e.moves[i];
        e.move(i, mv.x, mv.y);
    }
    return moved;
}

// Dynamic LDS: the keys of pl.lds_tokens tokens (and of the places behind the last), then the places that become free and those that
// move.
template <int WAVES>
__global__ __launch_bounds__(WAVES * 64) void evict_select_kernel(EvictGeom g, EvictPlan pl, int32_t *counts, int2 *moves) {
    constexpr int THREADS = WAVES * 64;
    __shared__ EvictLds<WAVES> sm;
    extern __shared__ __attribute__((aligned(16))) uint32_t dynamic[];
    const int z = blockIdx.x, b = z / g.Hkv, h = z % g.Hkv, tid = threadIdx.x;
    const int64_t room = min((int64_t)g.pages.table_width << g.pages.page_shift, (int64_t)g.slots);
    const int32_t *table = g.pages.table + (int64_t)b * g.pages.table_width;
    Eviction e;
    e.len = __builtin_amdgcn_readfirstlane(max(0, (int)min((int64_t)g.pages.tail_len[b], room)));
    e.keep = min(e.len, g.budget);
    e.rows = EvictRows{g.scores + b * g.ss[0] + h * g.ss[1], g.pos ? g.pos + b * g.ps[0] + h * g.ps[1] : nullptr,
                       (int)max((int64_t)(g.seen ? g.seen : g.pages.tail_len)[b] - g.recent, (int64_t)INT_MIN), g.sink};
    e.scores_out = g.scores_out + b * g.so[0] + h * g.so[1];
    e.pos_out = g.pos_out + b * g.po[0] + h * g.po[1];
    e.moves = moves + (int64_t)z * pl.moves;
    auto holes = [&] {
        bool hole = false;
        const int pages = (int)(((int64_t)e.len + (1 << g.pages.page_shift) - 1) >> g.pages.page_shift);
        for (int i = tid; i < pages; i += THREADS) hole |= table[i] < 0 || table[i] >= g.pages.n_pages;
        e.copy(tid, THREADS);
        return __syncthreads_or(hole) != 0;
    };
    static_assert(sizeof(sm) <= kEvictStatic, "what the plan leaves for it");
    int moved = 0;
    if (e.len == e.keep) {
        e.copy(tid, THREADS);
    } else if (e.len <= pl.lds_tokens) {
        moved = evict_in_lds<WAVES>(e, sm, dynamic, (uint16_t *)(dynamic + (pl.lds_tokens + THREADS)), tid, holes);
    } else if constexpr (WAVES == 16) {  // (fewer waves are for so few tokens that all keys fit)
        moved = evict_from_memory(e, sm, tid, holes);
    }
    if (e.keep > g.budget) e.copy(tid, THREADS);  // (a hole: all places)
    if (tid == 0) {
        counts[z] = moved;
        if (h == 0) g.len_out[b] = e.keep;
    }
    if (pl.in_one) {
        __syncthreads();
        move_rows(g, table, h, e.moves, moved, tid, THREADS);
    }
}

// (more moves than the launch has rows for: workgroups take several lots)
constexpr int kMoveRows = 16, kMoveWorkgroups = 1 << 16;  // of a lot; of a launch, at most, if every (sequence, KV head) gets one
__global__ __launch_bounds__(256) void evict_move_kernel(EvictGeom g, EvictPlan pl, const int32_t *counts, const int2 *moves) {
    const int z = blockIdx.y, b = z / g.Hkv, count = counts[z];
    for (int first = blockIdx.x * kMoveRows; first < count; first += gridDim.x * kMoveRows)
        move_rows(g, g.pages.table + (int64_t)b * g.pages.table_width, z % g.Hkv, moves + (int64_t)z * pl.moves + first, min(kMoveRows, count - first),
                  threadIdx.x, 256);
}

hipError_t launch_paged_evict(const EvictGeom &g, const EvictPlan &pl, void *ws, hipStream_t st) {
    int32_t *counts = (int32_t *)ws;
    int2 *moves = (int2 *)((char *)ws + pl.off_moves);
    const int Z = g.batch * g.Hkv;
    static DeviceOnce once;
    const hipError_t e0 = device_once(once, [] {
        return hipFuncSetAttribute((const void *)evict_select_kernel<16>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)kEvictDynamic);
    });
    if (e0 != hipSuccess) return e0;
    auto select = [&](auto kernel, int waves) { hipLaunchKernelGGL(kernel, dim3(Z), dim3(waves * 64), pl.lds_bytes, st, g, pl, counts, moves); };
    if (pl.waves == 4) select(evict_select_kernel<4>, 4);
    else if (pl.waves == 8) select(evict_select_kernel<8>, 8);
    else select(evict_select_kernel<16>, 16);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || pl.moves == 0 || pl.in_one) return e;
    const int lots = std::min((pl.moves + kMoveRows - 1) / kMoveRows, std::max(1, kMoveWorkgroups / Z));
    hipLaunchKernelGGL(evict_move_kernel, dim3(lots, Z), dim3(256), 0, st, g, pl, counts, moves);
    return hipGetLastError();
}

}  // namespace aha
