// Attention of a batch's new tokens over the prefixes that its sequences share and over their own tails in pages.
//
//   out = sum_j softmax_j(scale q . K_j) V_j
//
// in parts: a work item (shared_rows.h) forms sum_j 2^(x_j - m) V_j, sum_j 2^(x_j - m) and m over its keys, x = scale log2(e) q . K, in
// one pass with a running reference m; a row's parts are joined by a second launch.  A prefix's keys are read once for a tile of
// rows of all its sequences, which is what makes the products of a batch matrix products.  Tiles are of 32 rows here, of 128 and 256 in
// shared_wide.hip.
#include <limits.h>

#include "narrow_tile.h"
#include "shared_rows.h"

namespace aha {

// The waves' results of an item of 32 rows -> the workspace.
template <int D>
__device__ __forceinline__ void merge_waves(const SharedGeom &g, const SharedPlan &pl, const SharedItem &it, bool live_row, f32x16 (&O)[D / 32],
                                            float m, float s, char *smem, int lane, int wave, float *part_o, float2 *part_ms) {
    meet_waves<D>(
        it.row1 - it.row0, live_row, O, m, s, smem, lane, wave,
        [&](float M, float all) { part_ms[partial_index(g, pl, it.h, it.part, it.row0 + (lane & 31))] = make_float2(M, all); },
        [&](int q, int ch, const f32x4 &o) { *(f32x4 *)(part_o + partial_index(g, pl, it.h, it.part, it.row0 + q) * D + ch) = o; });
}

// ---- bf16, up to 32 rows ----
// Four waves take blocks of 32 keys in turn, each with all rows: a stream of keys and values, bound by memory.  Per block and
// wave: S^T = K Q^T and O^T += V^T P^T by v_mfma_f32_32x32x16_bf16, keys (channels) on M, rows on N, so that the accumulator elements of a
// lane are the probabilities that it supplies to the second product.  Keys go to registers, values to LDS, both a block ahead: 64 KB
// of requests per workgroup (d = 128), two of them per CU.  64 sequences of four prefixes of 4096 tokens, tails of up to 1001: 203 MB from memory (each prefix
// once: the second tile of its 64 rows finds it in the L2) in 52 us, 3.9 TB/s; what is missing of 4.8 are the items' starts, 4 to 6 us each, and the last
// tails.  8 sequences of one prefix of 2048: 9.4 us, a chain of five round trips.
// The weights are rounded to bf16 for the second product, as the matrix core takes them beside bf16 values (their sum is of the unrounded ones, in fp32):
// outputs are 0.0018 to 0.0023 from 64 bits, relative to their size, where a single rounding of the exact ones is 0.0017.  Weights in two
// parts would double that product.
template <int D>
__global__ __launch_bounds__(256, 2) void shared_narrow_kernel(SharedGeom g, SharedPlan pl, float *part_o, float2 *part_ms) {
    using A = NarrowRows<D>;
    constexpr int KS = D / 16, CB = D / 32;
    __shared__ __attribute__((aligned(1024))) char smem[narrow_lds<__bf16, D>()];
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), col = lane & 31, hf = lane >> 5;
    SharedItem it;
    if (!shared_item(g, pl, (int)blockIdx.x, 32, A::STEP, lane, it)) return;
    const SharedRow row(g, it, it.row0 + col);
    if (it.begin >= it.end) {  // no keys in this part
        if (tid < 32 && row.live) part_ms[partial_index(g, pl, it.h, it.part, it.row0 + tid)] = make_float2(-INFINITY, 0.f);
        return;
    }
    const SharedKeys<__bf16> keys(g, it);
    bf16x8 qf[KS];
    {
        const __bf16 *p = (const __bf16 *)g.q + row.b * g.qs[0] + row.hq * g.qs[1] + row.t * g.qs[2] + hf * 8;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            qf[ks] = *(const bf16x8 *)(p + ks * 16);
            if (!row.live) qf[ks] = bf16x8{};
        }
    }
    const float c_out = pl.c_out;
    const int limit = row.limit;
    f32x16 O[CB];
    float m, s;
    no_rows_yet(O, m, s);
    narrow_sweep<D>(keys, qf, limit, c_out, smem, lane, wave, O, m, s, [](int, const f32x16 &) {});
    merge_waves<D>(g, pl, it, row.live, O, m, s, smem, lane, wave, part_o, part_ms);
}

// ---- fp32 ----
// The same on v_mfma_f32_32x32x2_f32 (narrow_tile.h).
template <int D>
__global__ __launch_bounds__(256, 2) void shared_f32_kernel(SharedGeom g, SharedPlan pl, float *part_o, float2 *part_ms) {
    using A = NarrowRows<D>;
    constexpr int CB = D / 32;
    __shared__ __attribute__((aligned(16))) char smem[narrow_lds<float, D>()];
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), col = lane & 31, hf = lane >> 5;
    SharedItem it;
    if (!shared_item(g, pl, (int)blockIdx.x, 32, A::STEP, lane, it)) return;
    const SharedRow row(g, it, it.row0 + col);
    if (it.begin >= it.end) {
        if (tid < 32 && row.live) part_ms[partial_index(g, pl, it.h, it.part, it.row0 + tid)] = make_float2(-INFINITY, 0.f);
        return;
    }
    const SharedKeys<float> keys(g, it);
    float *sQ = (float *)smem;
    stage_f32_rows<D>(sQ, (const float *)g.q + row.b * g.qs[0] + row.hq * g.qs[1] + row.t * g.qs[2], row.live, lane, wave);
    __syncthreads();
    const float *sq = sQ + col * f32_ld(D) + 4 * hf;
    const float c_out = pl.c_out;
    const int limit = row.limit;
    f32x16 O[CB];
    float m, s;
    no_rows_yet(O, m, s);
    f32_sweep<D>(keys, sq, limit, c_out, lane, wave, O, m, s, [](int, const f32x16 &) {});
    merge_waves<D>(g, pl, it, row.live, O, m, s, smem, lane, wave, part_o, part_ms);
}

// ---- joining a row's parts ----
// A thread takes four channels of a row and every SP-th part, four parts' loads in flight at once (bound by their latency: one
// after the other, 33 parts took 23 us); the SP threads of a channel meet in LDS.  Parts without a key have a reference of -inf and no
// output; rows without a prefix have no prefix parts.
template <class T, int D, int SP>
__global__ __launch_bounds__(256) void shared_join_kernel(SharedGeom g, SharedPlan pl, const float *part_o, const float2 *part_ms) {
    constexpr int TPR = D / 4, ROWS = 256 / (TPR * SP), U = 4;
    const int per = rows_of_sequence(g), ch = threadIdx.x % TPR * 4, sp = threadIdx.x / TPR % SP;
    const int row = blockIdx.x * ROWS + threadIdx.x / (TPR * SP);
    const int h = blockIdx.y, b = min(row / per, g.batch - 1), at = row - b * per, gi = at / g.n, t = at - gi * g.n;
    const bool live = row < g.batch * per && t < fresh_of(g, b);
    JoinState x{-INFINITY, 0.f, f32x4{0.f, 0.f, 0.f, 0.f}};
    if (live) {
        int lo = 0, hi = g.n_prefixes;  // prefixes that begin at or before b
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (first_of(g, mid) <= b) lo = mid + 1; else hi = mid;
        }
        const bool ahead = lo > 0 && b < first_of(g, lo);
        const int p0 = ahead ? 0 : pl.prefix_parts, p1 = pl.prefix_parts + pl.tail_parts;
        const int64_t step = partial_index(g, pl, 0, 1, 0);
        for (int p = p0 + sp; p < p1; p += U * SP) {
            const int64_t i = partial_index(g, pl, h, p, row);
            float2 ms[U];
            f32x4 o[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {  // (past the last part: the first of these again)
                const int64_t j = p + u * SP < p1 ? i + u * SP * step : i;
                ms[u] = part_ms[j];
                o[u] = *(const f32x4 *)(part_o + j * D + ch);
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (p + u * SP < p1) x.add(ms[u].x, ms[u].y, o[u]);
        }
    }
    if constexpr (SP > 1) {
        __shared__ f32x4 s_o[256];
        __shared__ float2 s_ms[256];
        s_o[threadIdx.x] = x.o;
        s_ms[threadIdx.x] = make_float2(x.m, x.s);
        __syncthreads();
        if (sp) return;
#pragma unroll
        for (int u = 1; u < SP; ++u) x.add(s_ms[threadIdx.x + u * TPR].x, s_ms[threadIdx.x + u * TPR].y, s_o[threadIdx.x + u * TPR]);
    }
    if (!live) return;
    const float inv = x.s == 0.f ? 0.f : 1.f / x.s;
    store_output((T *)g.out + b * g.os[0] + (h * g.G + gi) * g.os[1] + t * g.os[2] + ch, x.o, inv);
    if (g.lse && ch == 0) g.lse[((int64_t)b * g.Hq + h * g.G + gi) * g.n + t] = x.s == 0.f ? -INFINITY : (x.m + log2f(x.s)) * kLn2;
}

template <class T, int D>
static hipError_t launch_shared_t(const SharedGeom &g, const SharedPlan &pl, void *ws, hipStream_t st) {
    float *part_o = (float *)ws;
    float2 *part_ms = (float2 *)((char *)ws + pl.off_ms);
    const int64_t items = pl.prefix_items + pl.tail_items;
    if (items > 0) {
        const hipError_t e = [&] {
            if constexpr (sizeof(T) == 4) {
                hipLaunchKernelGGL(shared_f32_kernel<D>, dim3((unsigned)items), dim3(256), 0, st, g, pl, part_o, part_ms);
                return hipGetLastError();
            } else {
                auto launch = [&](const SharedPlan &some, int rows) {
                    if (some.prefix_items + some.tail_items == 0) return hipSuccess;
                    if (rows > 32) return launch_shared_wide(g, some, rows, part_o, part_ms, st);
                    hipLaunchKernelGGL(shared_narrow_kernel<D>, dim3((unsigned)(some.prefix_items + some.tail_items)), dim3(256), 0, st, g, some,
                                       part_o, part_ms);
                    return hipGetLastError();
                };
                if (pl.prefix_rows == pl.tail_rows) return launch(pl, pl.tail_rows);
                SharedPlan some = pl;
                some.tail_items = 0;
                const hipError_t e1 = launch(some, pl.prefix_rows);
                if (e1 != hipSuccess) return e1;
                some = pl;
                some.prefix_items = 0;
                return launch(some, pl.tail_rows);
            }
        }();
        if (e != hipSuccess) return e;
    }
    const int64_t total = (int64_t)g.batch * g.G * g.n;
    auto join = [&](auto kernel, int rows) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)((total + rows - 1) / rows), g.Hkv), dim3(256), 0, st, g, pl, part_o, part_ms);
    };
    // (up to four parts are in flight at once anyway)
    if (pl.prefix_parts + pl.tail_parts <= 4) join(shared_join_kernel<T, D, 1>, 256 / (D / 4));
    else join(shared_join_kernel<T, D, 8>, 256 / (D / 4 * 8));
    return hipGetLastError();
}

hipError_t launch_shared_attention(const SharedGeom &g, const SharedPlan &pl, void *ws, hipStream_t st) {
    if (g.dtype == AHA_BF16) return g.d == 64 ? launch_shared_t<__bf16, 64>(g, pl, ws, st) : launch_shared_t<__bf16, 128>(g, pl, ws, st);
    return g.d == 64 ? launch_shared_t<float, 64>(g, pl, ws, st) : launch_shared_t<float, 128>(g, pl, ws, st);
}

}  // namespace aha
