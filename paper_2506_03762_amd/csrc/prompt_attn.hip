// Causal attention of packed prompts:
//
//   out_t = sum_{j <= t} softmax_j(scale q_t . K_j) V_j,   j in t's prompt
//
// in one pass over a row's keys with a running reference m.  A workgroup takes a tile of rows and all keys up to its last one, so that nothing has to be
// joined and a call is one launch.  Tiles have 32 rows (here; narrow_tile.h), fp32 also 16 (small_tile.h), 128 (prompt_mid.hip) or 256 (prompt_wide.hip);
// plan_prompt() chooses.
//
// Here four waves divide the keys of 32 rows of one head: the shortest chain for few rows, bound by the latency of its blocks of 128 keys (d = 64 0.7 us, 128
// 1.4 us, loads requested one block ahead) and the L1, but every tile reads its keys and values from the L2 again.  9 prompts of up to 777 tokens, 6 heads of 64
// over 2: 10.8 us.  fp32: one prompt of 512, 2 heads of 64, 9.9 us in 64 tiles of 16 rows, 15.2 in 32 of 32, each bound by the products of its rows; of
// 4096, 32 heads of 128 over 8, 1276 us, 108 TFLOP/s, 0.70 of a library's product of 8192^3.  With eight waves to a tile every shape was slower.
#include <limits.h>

#include "narrow_tile.h"
#include "prompt_tiles.h"
#include "small_tile.h"

namespace aha {

template <class T, int D, int ROWS, bool STAGED>
__global__ __launch_bounds__(256, (kNarrowWorkgroups<T, D>)) void prompt_narrow_kernel(PromptGeom g) {
    using A = Tile<T, D, ROWS>;
    __shared__ __attribute__((aligned(1024))) char smem[STAGED ? narrow_lds<T, D, true>() : A::lds];
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), col = lane % ROWS;
    PromptTile it;
    if (!prompt_tile(g, ROWS, g.item0 + (int)blockIdx.x, lane, it)) return;
    KeyPlaces<T> keys;
    keys.in_a_row((const T *)g.k + it.lo * g.ks[0] + it.h * g.ks[1], (const T *)g.v + it.lo * g.vs[0] + it.h * g.vs[1], g.ks[0], g.vs[0]);
    keys.begin = 0;
    keys.end = it.row1 - it.lo;
    const bool live = it.row0 + col < it.row1;
    const int token = min(it.row0 + col, it.row1 - 1), limit = token - it.lo;
    const T *q = (const T *)g.q + token * g.qs[0] + it.hq * g.qs[1];
    typename A::Out O;
    float m, s;
    no_rows_yet(O, m, s);
    if constexpr (sizeof(T) == 2) {
        bf16x8 qf[D / 16];
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) qf[ks] = *(const bf16x8 *)(q + (lane >> 5) * 8 + ks * 16);
        if constexpr (STAGED) staged_sweep<D>(keys, qf, limit, g.c_out, smem, lane, wave, O, m, s);
        else narrow_sweep<D>(keys, qf, limit, g.c_out, smem, lane, wave, O, m, s, [](int, const f32x16 &) {});
    } else if constexpr (ROWS == 16) {
        f32x4 qf[D / 16];
#pragma unroll
        for (int i = 0; i < D / 16; ++i) qf[i] = *(const f32x4 *)(q + A::first(lane) + 16 * i);
        f32_sweep16<D>(keys, qf, limit, g.c_out, lane, wave, O, m, s, [](int, const f32x8 &) {});
    } else {
        float *sQ = (float *)smem;
        stage_f32_rows<D>(sQ, q, true, lane, wave);
        __syncthreads();
        f32_sweep<D>(keys, sQ + col * f32_ld(D) + A::first(lane), limit, g.c_out, lane, wave, O, m, s, [](int, const f32x16 &) {});
    }
    const float *sums = (const float *)(smem + A::off_sums);
    meet_waves<D>(
        it.row1 - it.row0, live, O, m, s, smem, lane, wave,
        [&](float M, float all) {
            if (g.lse) g.lse[(int64_t)it.hq * g.tokens + token] = (M + log2f(all)) * kLn2;
        },
        [&](int r, int ch, const f32x4 &o) {
            store_output((T *)g.out + (it.row0 + r) * g.os[0] + it.hq * g.os[1] + ch, o, 1.f / sums[r]);
        });
}

template <class T, int D, int ROWS, bool STAGED>
static hipError_t launch_narrow(const PromptGeom &g, const PromptPlan &pl, hipStream_t st) {
    return launch_prompt_items(prompt_narrow_kernel<T, D, ROWS, STAGED>, g, pl, 0, st);
}

hipError_t launch_prompt_attention(const PromptGeom &g, const PromptPlan &pl, hipStream_t st) {
    if (pl.rows == 128) return launch_prompt_mid(g, pl, st);
    if (pl.rows > 32) return launch_prompt_wide(g, pl, st);
    if (g.dtype == AHA_BF16) {
        if (g.d == 128) return launch_narrow<__bf16, 128, 32, true>(g, pl, st);
        return pl.staged ? launch_narrow<__bf16, 64, 32, true>(g, pl, st) : launch_narrow<__bf16, 64, 32, false>(g, pl, st);
    }
    if (pl.rows == 16) return g.d == 64 ? launch_narrow<float, 64, 16, false>(g, pl, st) : launch_narrow<float, 128, 16, false>(g, pl, st);
    return g.d == 64 ? launch_narrow<float, 64, 32, false>(g, pl, st) : launch_narrow<float, 128, 32, false>(g, pl, st);
}

}  // namespace aha
