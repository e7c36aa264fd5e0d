// One pass of a tile of 16 query rows over a range of keys, fp32: as in narrow_tile.h, on v_mfma_f32_16x16x4_f32.
//
// The matrix core's fp32 rate is the same and half of a tile of 32 rows is empty where there are up to 16: a block of 32 keys and 64 channels takes 2048 cycles
// instead of 4096.  With more rows it reads the keys twice as often.  A lane's channels of a key row and a query row are 16 i + 4 (lane / 16) .. + 3, one of
// which is a contraction step's for its quarter of the wave; its weights are those of its row, lane % 16, and the keys 16 t + 4 (lane / 16) + r, element r of
// accumulator t, which the second product takes one element at a time, four keys to a step.
#pragma once

#include "narrow_tile.h"

namespace aha {

typedef float f32x8 __attribute__((ext_vector_type(8)));

// How a tile's logits lie: row lane % ROWS, logit v of a block of 32 is key(v) + first(lane).
template <int ROWS_>
struct TileRows {
    static constexpr int ROWS = ROWS_, N = ROWS / 2;
    static __device__ __forceinline__ int first(int lane) { return 4 * (lane / ROWS); }
    static constexpr __device__ __forceinline__ int key(int v) { return 256 / ROWS * (v >> 2) + (v & 3); }
};

template <int D>
__device__ __forceinline__ void no_rows_yet(f32x4 (&O)[D], float &m, float &s) {
    m = -INFINITY;
    s = 0.f;
#pragma unroll
    for (int cb = 0; cb < D; ++cb) O[cb] = f32x4{0.f, 0.f, 0.f, 0.f};
}
// `q`: the lane's chunks of its query row; else as narrow_sweep().
template <int D, class Keys, class Block>
__device__ __forceinline__ void f32_sweep16(const Keys &keys, const f32x4 (&q)[D / 16], int limit, float c_out, int lane, int wave, f32x4 (&O)[D / 16],
                                            float &m, float &s, Block block) {
    using R = TileRows<16>;
    constexpr int CB = D / 16, STEP = NarrowRows<D>::STEP;
    const int col = lane & 15, g = lane >> 4, limit_min = -reduce_lanes<1, 16>(-limit, OpMaxI{});
    int kb = keys.begin + wave * 32;
    if (kb >= keys.end) return;
    // (lane: what is known of key lane % 32; a block's values and the next one's keys are requested around its dots, its page a block earlier)
    int next_entry = keys.entry(kb + STEP + (lane & 31));
    auto here = keys.at(kb + (lane & 31), keys.entry(kb + (lane & 31)));
    auto row_of = [&](const float *mine, int key) {
        const uint64_t p = (uint64_t)(uintptr_t)mine;
        return (const float *)(((uint64_t)__shfl((uint32_t)(p >> 32), key) << 32) | __shfl((uint32_t)p, key));
    };
    f32x4 a[2][CB];
    auto load_keys = [&] {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const float *k = row_of(here.k, 16 * t + col) + 4 * g;
#pragma unroll
            for (int i = 0; i < CB; ++i) a[t][i] = load_global<f32x4>(k + 16 * i);
        }
    };
    load_keys();
    for (; kb < keys.end; kb += STEP) {
        const uint32_t there = (uint32_t)__builtin_amdgcn_ballot_w64(here.there);
        float v_row[R::N][CB];
#pragma unroll
        for (int v = 0; v < R::N; ++v) {
            const float *vr = row_of(here.v, R::key(v) + 4 * g) + col;
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) v_row[v][cb] = load_global<float>(vr + cb * 16);
        }
        here = keys.at(kb + STEP + (lane & 31), next_entry);
        next_entry = keys.entry(kb + 2 * STEP + (lane & 31));
        __builtin_amdgcn_sched_barrier(0);
        // (two chains to a dot, D / 8 products each as in narrow_tile.h)
        f32x4 dot[2][2];
#pragma unroll
        for (int t = 0; t < 2; ++t) dot[t][0] = dot[t][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < CB; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int t = 0; t < 2; ++t) dot[t][e & 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[t][i][e], q[i][e], dot[t][e & 1], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
        load_keys();
        __builtin_amdgcn_sched_barrier(0);
        f32x8 acc;
#pragma unroll
        for (int v = 0; v < R::N; ++v) acc[v] = dot[v >> 2][0][v & 3] + dot[v >> 2][1][v & 3];
        if (there != 0xffffffffu || kb + 31 > limit_min) {
#pragma unroll
            for (int v = 0; v < R::N; ++v) {
                const int at = R::key(v) + 4 * g;
                if (kb + at > limit || !((there >> at) & 1)) acc[v] = -INFINITY;
            }
        }
        block(kb, acc);
        float amax = -INFINITY;
#pragma unroll
        for (int v = 0; v < R::N; ++v) amax = fmaxf(amax, acc[v]);
        amax = reduce_lanes<16, 64>(amax, OpMax{});
        const float mn = fmaxf(m, amax * c_out), mref = mn == -INFINITY ? 0.f : mn, corr = fast_exp2(m - mref);
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int v = 0; v < R::N; ++v) {
            acc[v] = fast_exp2(fmaf(acc[v], c_out, -mref));
            sum[v & 1] += acc[v];
        }
        s = s * corr + (sum[0] + sum[1]);
        m = mn;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) O[cb] *= corr;
#pragma unroll
        for (int v = 0; v < R::N; ++v)
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) O[cb] = __builtin_amdgcn_mfma_f32_16x16x4f32(v_row[v][cb], acc[v], O[cb], 0, 0, 0);
    }
}

// The waves' results meet, as in narrow_tile.h: all channels at a time.
template <int D>
struct SmallMerge {
    static constexpr int WAVES = 4, LDO = D + 4;
    static constexpr size_t o_bytes = (size_t)WAVES * 16 * LDO * 4, off_sums = o_bytes + (size_t)WAVES * 16 * 8, bytes = off_sums + 16 * 4;
};
template <int D, class Row, class Store>
__device__ __forceinline__ void meet_waves(int rows, bool live_row, f32x4 (&O)[D / 16], float m, float s, char *smem, int lane, int wave, Row row,
                                           Store store) {
    using A = SmallMerge<D>;
    constexpr int CPR = D / 4;
    const int tid = wave * 64 + lane, col = lane & 15, g = lane >> 4;
    float2 *sMS = (float2 *)(smem + A::o_bytes);
    const float sc = reduce_lanes<16, 64>(s, OpSum{});
    if (lane < 16) sMS[wave * 16 + lane] = make_float2(m, sc);
    const uint32_t live = (uint32_t)__builtin_amdgcn_ballot_w64(live_row) & 0xffffu;
    __syncthreads();
    float M = -INFINITY, all = 0.f;
#pragma unroll
    for (int w = 0; w < A::WAVES; ++w) M = fmaxf(M, sMS[w * 16 + col].x);
    const float mref = M == -INFINITY ? 0.f : M, f = fast_exp2(m - mref);
#pragma unroll
    for (int w = 0; w < A::WAVES; ++w) all = fmaf(fast_exp2(sMS[w * 16 + col].x - mref), sMS[w * 16 + col].y, all);
    if (tid < 16) ((float *)(smem + A::off_sums))[col] = all;
    if (tid < 16 && live_row) row(M, all);
    if (live_row) {
        float *sO = (float *)smem + (wave * 16 + col) * A::LDO + 4 * g;
#pragma unroll
        for (int cb = 0; cb < D / 16; ++cb) *(f32x4 *)(sO + 16 * cb) = O[cb] * f;
    }
    __syncthreads();
    for (int i = tid; i < rows * CPR; i += 256) {
        const int q = i / CPR, ch = i % CPR * 4;
        if (!((live >> q) & 1)) continue;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < A::WAVES; ++w) o += *(const f32x4 *)((const float *)smem + (w * 16 + q) * A::LDO + ch);
        store(q, ch, o);
    }
}

// What a kernel of these tiles takes by its number of rows.
template <class T, int D, int ROWS>
struct Tile : TileRows<ROWS> {
    static constexpr int CB = D / 32;
    typedef f32x16 Out[CB];
    static constexpr size_t lds = narrow_lds<T, D>(), off_sums = WaveMerge<D>::off_sums;
};
template <class T, int D>
struct Tile<T, D, 16> : TileRows<16> {
    static constexpr int CB = D / 16;
    typedef f32x4 Out[CB];
    static constexpr size_t lds = SmallMerge<D>::bytes, off_sums = SmallMerge<D>::off_sums;
};

}  // namespace aha
