// Attention of one new token of every sequence over its paged cache, and the running scores of the cached tokens:
//
//   out = sum_j softmax_j(scale q . K_j) V_j        F_j += sum_g softmax_j(lambda q_g . K_j)
//
// in two launches.  The first takes the keys of a (sequence, KV head) in parts: the rows of its query heads, padded to tiles of 32 (narrow_tile.h; fp32 with up to 16
// heads one of 16, small_tile.h), in one pass over the part's keys and values, which leaves the products, a partial output and the sums of both softmaxes, relative
// to references of their own, in the workspace.  The second joins the parts: outputs by row, scores by range of keys.  Where there is one part, its
// workgroup does that itself (plan_paged() says when).
//
// Bound by memory: keys and values are read once, for all query heads of their KV head, and two operations per element and head are far below what the
// matrix core gives.  64 caches of up to 4096 tokens, 8 heads of 128: 670 MB in 145 us, 4.6 TB/s (a copy reaches 4.95), joining 12 more; one cache
// of 131072 tokens 540 MB in 113 us, 4.75 TB/s, joining 11; 8 caches of 2049 tokens 18.5 + 4.5, of which 14 are the 67 MB.
// Small caches are a chain: 8 of 64 tokens 9 us, 5 of them the launch's.
#include <limits.h>

#include "small_tile.h"

namespace aha {

// The tokens of sequence b.
__device__ __forceinline__ int tokens_of(const PagedGeom &g, int b) {
    const int64_t room = (int64_t)g.pages.table_width << g.pages.page_shift;
    return max(0, (int)min((int64_t)g.pages.tail_len[b], g.slots > 0 ? min(room, (int64_t)g.slots) : room));
}
// Scale of the accumulated weights, times log2(e); above 0, with which a masked product, -inf, is no number otherwise.
__device__ __forceinline__ float score_scale(const PagedGeom &g, int b) {
    const int c = max(1, (g.seen ? g.seen : g.pages.tail_len)[b]);
    return fmaxf(row_scale_log2(g.scale_mode, g.fixed_scale, g.lambda_floor, c, g.budget, g.d), 0x1p-149f);
}
// Number of the partial result of row gi of (sequence, KV head) z.
__device__ __forceinline__ int64_t paged_partial(const PagedGeom &g, const PagedPlan &pl, int z, int part, int gi) {
    return ((int64_t)z * pl.parts + part) * g.G + gi;
}

// The scores of four tokens from j0 on: `dot` the products of the first U rows, `score` and `page` what the tokens have (places past the last one: anything),
// `norm` reference and 1 / sum of every row.
constexpr int kScoreRows = 4;  // rows whose products are in flight at once
struct ScoreLoads {
    f32x4 dot[kScoreRows];
    float score[4];
    int page[4];
    // (nothing of the sequence's length: places lie within the workspace's rows, the table and the scores wherever its end is)
    __device__ __forceinline__ void request(const PagedGeom &g, const float *x, int64_t ld, const float *F, const int32_t *table, int at) {
#pragma unroll
        for (int u = 0; u < kScoreRows; ++u) dot[u] = *(const f32x4 *)(x + min(u, g.G - 1) * ld + at);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            score[i] = F[min(at + i, g.slots - 1)];
            page[i] = table[min((at + i) >> g.pages.page_shift, g.pages.table_width - 1)];
        }
    }
    __device__ __forceinline__ void add(const PagedGeom &g, const float *x, int64_t ld, float *F, int32_t *pos, int at, int j0, int len, int seen, float lam,
                                        const float2 *norm) {
        float w[4] = {0.f, 0.f, 0.f, 0.f};
        for (int g0 = 0; g0 < g.G; g0 += kScoreRows) {
            if (g0) {
#pragma unroll
                for (int u = 0; u < kScoreRows; ++u) dot[u] = *(const f32x4 *)(x + min(g0 + u, g.G - 1) * ld + at);
            }
#pragma unroll
            for (int u = 0; u < kScoreRows; ++u)
                if (g0 + u < g.G) {
                    const float2 n = norm[g0 + u];
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[i] += fast_exp2(fmaf(dot[u][i], lam, -n.x)) * n.y;
                }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int j = j0 + i;
            if (j >= len) break;
            const bool there = page[i] >= 0 && page[i] < g.pages.n_pages;
            if (j == len - 1) {
                F[j] = there ? w[i] : 0.f;
                if (pos) pos[j] = seen - 1;
            } else if (there) {
                F[j] = score[i] + w[i];
            }
        }
    }
};
// Reference and 1 / sum of a row's weights (NaN stays).
__device__ __forceinline__ float2 score_norm(float ref, float all) { return make_float2(ref, all > 0.f ? 1.f / all : all == 0.f ? 0.f : all); }

// ONE: all keys are one part, whose outputs and scores are formed here.
template <class T, int D, int ROWS, bool ONE>
__global__ __launch_bounds__(256, (kNarrowWorkgroups<T, D>)) void paged_part_kernel(PagedGeom g, PagedPlan pl, float *part_o, float2 *part_ms,
                                                                              float2 *part_ms2, float *dots) {
    using A = Tile<T, D, ROWS>;
    constexpr int STEP = NarrowRows<D>::STEP;
    __shared__ __attribute__((aligned(1024))) char smem[A::lds];
    __shared__ float2 s_ms2[4][ROWS], s_norm[ROWS];
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), col = lane % ROWS;
    // (sequence, KV head) by part by tile
    const int id = blockIdx.x, tile = id % pl.tiles, part = id / pl.tiles % pl.parts, z = id / pl.tiles / pl.parts;
    const int b = z / g.Hkv, h = z % g.Hkv, row0 = tile * ROWS, rows = min(ROWS, g.G - row0);
    const int len = uniform(tokens_of(g, b)), steps = (len + STEP - 1) / STEP;
    const bool live = col < rows;
    const int gi = row0 + min(col, rows - 1), hq = h * g.G + gi;
    KeyPlaces<T> keys;
    keys.in_pages(g.pages, g.kt, g.vt, b, h);
    keys.begin = (int)((int64_t)part * steps / pl.parts) * STEP;
    keys.end = min(len, (int)((int64_t)(part + 1) * steps / pl.parts) * STEP);
    if (keys.begin >= keys.end) {
        if constexpr (ONE) {
            for (int i = tid; i < rows * (D / 4); i += 256)
                store_output((T *)g.out + b * g.os[0] + (h * g.G + i / (D / 4)) * g.os[1] + i % (D / 4) * 4, f32x4{0.f, 0.f, 0.f, 0.f}, 0.f);
            if (tid < rows && g.lse) g.lse[(int64_t)b * g.Hq + h * g.G + tid] = -INFINITY;
        } else if (tid < rows) {
            part_ms[paged_partial(g, pl, z, part, row0 + tid)] = make_float2(-INFINITY, 0.f);
            if (dots) part_ms2[paged_partial(g, pl, z, part, row0 + tid)] = make_float2(-INFINITY, 0.f);
        }
        return;
    }
    const T *q = (const T *)g.q + b * g.qs[0] + hq * g.qs[1];
    float *to = dots + ((int64_t)b * g.Hq + hq) * pl.ld + A::first(lane);
    const float lam = dots ? score_scale(g, b) : 0.f;
    float m2 = -INFINITY, s2 = 0.f;
    auto block = [&](int kb, const auto &acc) {
        if (!dots) return;
        if (live) {
#pragma unroll
            for (int v = 0; v < A::N; v += 4) *(f32x4 *)(to + kb + A::key(v)) = f32x4{acc[v], acc[v + 1], acc[v + 2], acc[v + 3]};
        }
        float top = -INFINITY;
#pragma unroll
        for (int v = 0; v < A::N; ++v) top = fmaxf(top, acc[v]);
        const float mn = fmaxf(m2, top * lam), ref = mn == -INFINITY ? 0.f : mn;
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int v = 0; v < A::N; ++v) sum[v & 3] += fast_exp2(fmaf(acc[v], lam, -ref));
        s2 = s2 * fast_exp2(m2 - ref) + ((sum[0] + sum[1]) + (sum[2] + sum[3]));
        m2 = mn;
    };
    typename A::Out O;
    float m, s;
    no_rows_yet(O, m, s);
    if constexpr (sizeof(T) == 2) {
        bf16x8 qf[D / 16];
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
            qf[ks] = *(const bf16x8 *)(q + (lane >> 5) * 8 + ks * 16);
            if (!live) qf[ks] = bf16x8{};
        }
        narrow_sweep<D, true>(keys, qf, INT_MAX, g.c_out, smem, lane, wave, O, m, s, block);
    } else if constexpr (ROWS == 16) {
        f32x4 qf[D / 16];
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            qf[i] = *(const f32x4 *)(q + A::first(lane) + 16 * i);
            if (!live) qf[i] = f32x4{};
        }
        f32_sweep16<D>(keys, qf, INT_MAX, g.c_out, lane, wave, O, m, s, block);
    } else {
        float *sQ = (float *)smem;
        stage_f32_rows<D>(sQ, q, live, lane, wave);
        __syncthreads();
        f32_sweep<D>(keys, sQ + col * f32_ld(D) + A::first(lane), INT_MAX, g.c_out, lane, wave, O, m, s, block);
    }
    if (dots) {  // the sums of a row's lanes, later those of the waves
        const float M = reduce_lanes<ROWS, 64>(m2, OpMax{}), ref = M == -INFINITY ? 0.f : M;
        const float all = reduce_lanes<ROWS, 64>(s2 * fast_exp2(m2 - ref), OpSum{});
        if (lane < ROWS) s_ms2[wave][lane] = make_float2(M, all);
    }
    const float *sums = (const float *)(smem + A::off_sums);
    meet_waves<D>(
        rows, live, O, m, s, smem, lane, wave,
        [&](float M, float all) {
            const int64_t p = paged_partial(g, pl, z, part, gi);
            if constexpr (!ONE) part_ms[p] = make_float2(M, all);
            else if (g.lse) g.lse[(int64_t)b * g.Hq + hq] = all == 0.f ? -INFINITY : (M + log2f(all)) * kLn2;
            if (!dots) return;
            float M2 = -INFINITY, all2 = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) M2 = fmaxf(M2, s_ms2[w][col].x);
            const float ref = M2 == -INFINITY ? 0.f : M2;
#pragma unroll
            for (int w = 0; w < 4; ++w) all2 = fmaf(fast_exp2(s_ms2[w][col].x - ref), s_ms2[w][col].y, all2);
            if constexpr (ONE) s_norm[col] = score_norm(ref, all2);
            else part_ms2[p] = make_float2(M2, all2);
        },
        [&](int r, int ch, const f32x4 &o) {
            if constexpr (ONE) {
                const float all = sums[r];
                store_output((T *)g.out + b * g.os[0] + (h * g.G + r) * g.os[1] + ch, o, all == 0.f ? 0.f : 1.f / all);
            } else {
                *(f32x4 *)(part_o + paged_partial(g, pl, z, part, row0 + r) * D + ch) = o;
            }
        });
    if constexpr (ONE) {
        if (!dots) return;
        __syncthreads();  // the products of all waves, and s_norm
        const float *x = dots + ((int64_t)b * g.Hq + (int64_t)h * g.G) * pl.ld;
        const int seen = (g.seen ? g.seen : g.pages.tail_len)[b];
        for (int j0 = 4 * tid; j0 < len; j0 += 1024) {
            float *F = g.scores + b * g.ss[0] + h * g.ss[1];
            ScoreLoads l;
            l.request(g, x, pl.ld, F, keys.table, j0);
            l.add(g, x, pl.ld, F, g.pos ? g.pos + b * g.ps[0] + h * g.ps[1] : nullptr, j0, j0, len, seen, lam, s_norm);
        }
    }
}

// ---- joining ----
// Workgroups of a (sequence, KV head): the first `g.G` / rows ones join output rows, the others take kJoinKeys keys of the scores each.
constexpr int kJoinKeys = 1024, kMaxGroup = 1024;
template <class T, int D, int SP>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedGeom g, PagedPlan pl, const float *part_o, const float2 *part_ms,
                                                         const float2 *part_ms2, const float *dots) {
    constexpr int TPR = D / 4, ROWS = 256 / (TPR * SP), U = 4;
    const int z = blockIdx.y, b = z / g.Hkv, h = z % g.Hkv, tid = threadIdx.x, out_wgs = (g.G + ROWS - 1) / ROWS;
    if ((int)blockIdx.x < out_wgs) {
        const int ch = tid % TPR * 4, sp = tid / TPR % SP, gi = blockIdx.x * ROWS + tid / (TPR * SP);
        JoinState x{-INFINITY, 0.f, f32x4{0.f, 0.f, 0.f, 0.f}};
        if (gi < g.G) {
            for (int p = sp; p < pl.parts; p += U * SP) {
                float2 ms[U];
                f32x4 o[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {  // (past the last part: the first of these again)
                    const int64_t i = paged_partial(g, pl, z, p + u * SP < pl.parts ? p + u * SP : p, gi);
                    ms[u] = part_ms[i];
                    o[u] = *(const f32x4 *)(part_o + i * D + ch);
                }
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (p + u * SP < pl.parts) x.add(ms[u].x, ms[u].y, o[u]);
            }
        }
        if constexpr (SP > 1) {
            __shared__ f32x4 s_o[256];
            __shared__ float2 s_ms[256];
            s_o[tid] = x.o;
            s_ms[tid] = make_float2(x.m, x.s);
            __syncthreads();
            if (sp) return;
#pragma unroll
            for (int u = 1; u < SP; ++u) x.add(s_ms[tid + u * TPR].x, s_ms[tid + u * TPR].y, s_o[tid + u * TPR]);
        }
        if (gi >= g.G) return;
        const int hq = h * g.G + gi;
        store_output((T *)g.out + b * g.os[0] + hq * g.os[1] + ch, x.o, x.s == 0.f ? 0.f : 1.f / x.s);
        if (g.lse && ch == 0) g.lse[(int64_t)b * g.Hq + hq] = x.s == 0.f ? -INFINITY : (x.m + log2f(x.s)) * kLn2;
        return;
    }
    // ---- scores: a thread takes four tokens (requested before anything of the sequence is known) ----
    __shared__ float2 norm[kMaxGroup];
    const int lane = tid & 63, j0 = (blockIdx.x - out_wgs) * kJoinKeys + 4 * tid, at = min(j0, (int)pl.ld - 4);
    const float *x = dots + ((int64_t)b * g.Hq + (int64_t)h * g.G) * pl.ld;
    float *F = g.scores + b * g.ss[0] + h * g.ss[1];
    ScoreLoads l;
    l.request(g, x, pl.ld, F, g.pages.table + (int64_t)b * g.pages.table_width, at);
    const int len = tokens_of(g, b), seen = (g.seen ? g.seen : g.pages.tail_len)[b];
    if ((blockIdx.x - out_wgs) * kJoinKeys >= len) return;
    for (int gi = tid >> 6; gi < g.G; gi += 4) {  // (up to 64 parts, one per lane)
        const float2 ms = lane < pl.parts ? part_ms2[paged_partial(g, pl, z, lane, gi)] : make_float2(-INFINITY, 0.f);
        const float M = wave_max(ms.x), ref = M == -INFINITY ? 0.f : M, all = wave_sum(fast_exp2(ms.x - ref) * ms.y);
        if (lane == 0) norm[gi] = score_norm(ref, all);
    }
    __syncthreads();
    l.add(g, x, pl.ld, F, g.pos ? g.pos + b * g.ps[0] + h * g.ps[1] : nullptr, at, j0, len, seen, score_scale(g, b), norm);
}

template <class T, int D, int ROWS>
static hipError_t launch_parts(const PagedGeom &g, const PagedPlan &pl, float *part_o, float2 *part_ms, float2 *part_ms2, float *dots, hipStream_t st) {
    if (pl.one) hipLaunchKernelGGL((paged_part_kernel<T, D, ROWS, true>), dim3((unsigned)pl.items), dim3(256), 0, st, g, pl, part_o, part_ms, part_ms2, dots);
    else hipLaunchKernelGGL((paged_part_kernel<T, D, ROWS, false>), dim3((unsigned)pl.items), dim3(256), 0, st, g, pl, part_o, part_ms, part_ms2, dots);
    return hipGetLastError();
}
template <class T, int D>
static hipError_t launch_paged_t(const PagedGeom &g, const PagedPlan &pl, void *ws, hipStream_t st) {
    float *part_o = (float *)ws, *dots = g.slots > 0 ? (float *)((char *)ws + pl.off_dots) : nullptr;
    float2 *part_ms = (float2 *)((char *)ws + pl.off_ms), *part_ms2 = (float2 *)((char *)ws + pl.off_ms2);
    auto launch = launch_parts<T, D, 32>;
    if constexpr (sizeof(T) == 4)
        if (pl.rows == 16) launch = launch_parts<T, D, 16>;
    const hipError_t e = launch(g, pl, part_o, part_ms, part_ms2, dots, st);
    if (e != hipSuccess || pl.one) return e;
    const int score_wgs = g.slots > 0 ? (int)((pl.ld + kJoinKeys - 1) / kJoinKeys) : 0;
    auto join = [&](auto kernel, int rows) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)((g.G + rows - 1) / rows + score_wgs), g.batch * g.Hkv), dim3(256), 0, st, g, pl, part_o, part_ms,
                           part_ms2, dots);
    };
    // (up to four parts are in flight at once anyway)
    if (pl.parts <= 4) join(paged_join_kernel<T, D, 1>, 256 / (D / 4));
    else join(paged_join_kernel<T, D, 8>, 256 / (D / 4 * 8));
    return hipGetLastError();
}

hipError_t launch_paged_attention(const PagedGeom &g, const PagedPlan &pl, void *ws, hipStream_t st) {
    if (g.dtype == AHA_BF16) return g.d == 64 ? launch_paged_t<__bf16, 64>(g, pl, ws, st) : launch_paged_t<__bf16, 128>(g, pl, ws, st);
    return g.d == 64 ? launch_paged_t<float, 64>(g, pl, ws, st) : launch_paged_t<float, 128>(g, pl, ws, st);
}

}  // namespace aha
