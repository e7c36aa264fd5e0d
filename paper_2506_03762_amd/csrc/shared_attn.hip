// Attention of a batch's new tokens over the prefixes that its sequences share and over their own tails in pages.
//
//   out = sum_j softmax_j(scale q . K_j) V_j
//
// in parts: a work item (shared_rows.h) forms sum_j 2^(x_j - m) V_j, sum_j 2^(x_j - m) and m over its keys, x = scale log2(e) q . K, in
// one pass with a running reference m; a row's parts are joined by a second launch.  A prefix's keys are read once for a tile of
// rows of all its sequences, which is what makes the products of a batch matrix products.  Tiles are of 32 rows here, of 128 and 256 in
// shared_wide.hip.
#include <limits.h>

#include "f32_tile.h"
#include "shared_rows.h"
#include "value_rows.h"

namespace aha {

constexpr float kRefSlack = 8.f;  // log2 units that a reference may lie below the running maximum
constexpr float kLn2 = 0.69314718055994531f;

// ---- the waves' results of an item of 32 rows -> the workspace ----
// Lane: row lane % 32, accumulator element v of channel block cb: channel 32 cb + 8 (v / 4) + 4 (lane / 32) + v % 4.  Every wave scales
// its output to the largest reference, half of the channels at a time meet in LDS, and a thread adds four channels of the
// waves' rows (with a channel at a time and its weights formed there, 4 us of an item's 10; so 1).
template <int D>
struct WaveMerge {
    static constexpr int WAVES = 4, HC = D / 2, LDO = HC + 4;  // channels at a time, floats of a row
    static constexpr size_t o_bytes = (size_t)WAVES * 32 * LDO * 4, bytes = o_bytes + (size_t)WAVES * 32 * 8;
};
template <int D>
__device__ __forceinline__ void merge_waves(const SharedGeom &g, const SharedPlan &pl, const SharedItem &it, bool live_row, f32x16 (&O)[D / 32],
                                            float m, float s, char *smem, int lane, int wave, float *part_o, float2 *part_ms) {
    using A = WaveMerge<D>;
    constexpr int CB = D / 32, CPR = A::HC / 4;
    const int tid = wave * 64 + lane, col = lane & 31, hf = lane >> 5, rows = it.row1 - it.row0;
    float2 *sMS = (float2 *)(smem + A::o_bytes);
    __syncthreads();  // what the LDS held is done with
    const float sc = combine_lane_xor<32>(s, OpSum{});
    if (lane < 32) sMS[wave * 32 + lane] = make_float2(m, sc);
    const uint32_t live = (uint32_t)__builtin_amdgcn_ballot_w64(live_row);
    __syncthreads();
    float M = -INFINITY, all = 0.f;
#pragma unroll
    for (int w = 0; w < A::WAVES; ++w) M = fmaxf(M, sMS[w * 32 + col].x);
    const float mref = M == -INFINITY ? 0.f : M, f = fast_exp2(m - mref);
#pragma unroll
    for (int w = 0; w < A::WAVES; ++w) all = fmaf(fast_exp2(sMS[w * 32 + col].x - mref), sMS[w * 32 + col].y, all);
    if (tid < 32 && live_row) part_ms[partial_index(g, pl, it.h, it.part, it.row0 + col)] = make_float2(M, all);
#pragma unroll
    for (int hc = 0; hc < 2; ++hc) {
        float *sO = (float *)smem + (wave * 32 + col) * A::LDO + 4 * hf;
        if (hc) __syncthreads();
        if (live_row) {
#pragma unroll
            for (int cb = 0; cb < CB / 2; ++cb)
#pragma unroll
                for (int v = 0; v < 16; v += 4) {
                    const f32x16 &x = O[hc * (CB / 2) + cb];
                    *(f32x4 *)(sO + cb * 32 + 2 * v) = f32x4{x[v] * f, x[v + 1] * f, x[v + 2] * f, x[v + 3] * f};
                }
        }
        __syncthreads();
        for (int i = tid; i < rows * CPR; i += 256) {
            const int q = i / CPR, ch = i % CPR * 4;
            if (!((live >> q) & 1)) continue;
            f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < A::WAVES; ++w) o += *(const f32x4 *)((const float *)smem + (w * 32 + q) * A::LDO + ch);
            *(f32x4 *)(part_o + partial_index(g, pl, it.h, it.part, it.row0 + q) * D + hc * A::HC + ch) = o;
        }
    }
}

// ---- bf16, up to 32 rows ----
// Four waves take blocks of 32 keys in turn, each with all rows: a stream of keys and values, bound by memory.  Per block and
// wave: S^T = K Q^T and O^T += V^T P^T by v_mfma_f32_32x32x16_bf16, keys (channels) on M, rows on N, so that the accumulator elements of a
// lane are the probabilities that it supplies to the second product.  Keys go to registers, values to LDS, both a block ahead: 64 KB
// of requests per workgroup (d = 128), two of them per CU.  64 sequences of four prefixes of 4096 tokens, tails of up to 1001: 203 MB from memory (each prefix once:
// the second tile of its 64 rows finds it in the L2) in 52 us, 3.9 TB/s; what is missing of 4.8 are the items' starts, 4 to 6 us each, and the last
// tails.  8 sequences of one prefix of 2048: 9.4 us, a chain of five round trips.
// The weights are rounded to bf16 for the second product, as the matrix core takes them beside bf16 values (their sum is of the unrounded ones, in fp32):
// outputs are 0.0018 to 0.0023 from 64 bits, relative to their size, where a single rounding of the exact ones is 0.0017.  Weights in two
// parts would double that product.
template <int D>
struct NarrowAttn {
    static constexpr int WAVES = 4, STEP = 32 * WAVES, CPR = D / 8, RPI = 64 / CPR, NI = 32 / RPI;
    static constexpr size_t v_bytes = 32 * D * 2;   // a block's value rows
    static constexpr size_t stage_bytes = 2 * WAVES * v_bytes;
    static constexpr size_t bytes = stage_bytes > WaveMerge<D>::bytes ? stage_bytes : WaveMerge<D>::bytes;
};
template <int D>
__global__ __launch_bounds__(256, 2) void shared_narrow_kernel(SharedGeom g, SharedPlan pl, float *part_o, float2 *part_ms) {
    using A = NarrowAttn<D>;
    constexpr int KS = D / 16, CB = D / 32;
    __shared__ __attribute__((aligned(1024))) char smem[A::bytes];
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
    const int limit = row.limit, limit_min = -reduce_lanes<1, 32>(-limit, OpMaxI{});

    // Value rows of a block -> LDS, chunks permuted on the way (value_rows.h); loads are assembly, waited for by hand.
    const uint32_t lds0 = uniform((int)((uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)smem + wave * 2 * (int)A::v_bytes));
    const int lr = lane / A::CPR, chunk = (lane % A::CPR) ^ value_chunk_swizzle<D>(lr);
    auto request_values = [&](const __bf16 *v, int buf) {  // v: this lane's row lane % 32
        const uint64_t mine = (uint64_t)(uintptr_t)v;
#pragma unroll
        for (int j = 0; j < A::NI; ++j) {
            const int from = j * A::RPI + lr;
            const uint32_t lo = __shfl((uint32_t)mine, from), hi = __shfl((uint32_t)(mine >> 32), from);
            const uint64_t src = (((uint64_t)hi << 32) | lo) + chunk * 16;
            asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
                         :
                         : "v"(src), "s"(lds0 + buf * (int)A::v_bytes + j * 1024)
                         : "memory");
        }
    };
    bf16x8 a[KS];
    auto load_keys = [&](const __bf16 *k) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) a[ks] = *(const bf16x8 *)(k + hf * 8 + ks * 16);
    };

    f32x16 O[CB];
    float m = -INFINITY, s = 0.f;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int v = 0; v < 16; ++v) O[cb][v] = 0.f;
    int kb = it.begin + wave * 32;
    int next_entry = keys.entry(kb + A::STEP + col);
    auto here = keys.at(kb + col, keys.entry(kb + col));
    request_values(here.v, 0);
    load_keys(here.k);
    for (int buf = 0; kb < it.end; kb += A::STEP, buf ^= 1) {
        __builtin_amdgcn_sched_barrier(0);
        wait_loads<0>();                                   // this block's keys and values are here,
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // and the last block's values have been read
        const uint32_t there = (uint32_t)__builtin_amdgcn_ballot_w64(here.there);  // (lanes 0 .. 31)
        here = keys.at(kb + A::STEP + col, next_entry);
        next_entry = keys.entry(kb + 2 * A::STEP + col);
        request_values(here.v, buf ^ 1);
        f32x16 acc;
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[v] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[ks], qf[ks], acc, 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
        load_keys(here.k);
        __builtin_amdgcn_sched_barrier(0);
        if (there != 0xffffffffu || kb + 31 > limit_min) {
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int at = 8 * (v >> 2) + 4 * hf + (v & 3);
                if (kb + at > limit || !((there >> at) & 1)) acc[v] = -INFINITY;
            }
        }
        float amax = -INFINITY;
#pragma unroll
        for (int v = 0; v < 16; ++v) amax = fmaxf(amax, acc[v]);
        amax = combine_lane_xor<32>(amax, OpMax{});
        // (the reference follows the running maximum lazily: it moves when a block's exceeds it by more than kRefSlack)
        const float bm = amax * c_out;
        const float mn = bm > m + kRefSlack ? bm : m;
        const float mref = mn == -INFINITY ? 0.f : mn;
        const float corr = fast_exp2(m - mref);
        float sum[2] = {0.f, 0.f};
        bf16x8 pf[2];
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float pr = fast_exp2(fmaf(acc[8 * ks + e], c_out, -mref));
                sum[e & 1] += pr;
                pf[ks][e] = (__bf16)pr;
            }
        s = s * corr + (sum[0] + sum[1]);
        m = mn;
        if (__builtin_amdgcn_ballot_w64(corr != 1.f) != 0) {
#pragma unroll
            for (int cb = 0; cb < CB; ++cb)
#pragma unroll
                for (int v = 0; v < 16; ++v) O[cb][v] *= corr;
        }
        const __bf16 *sV = (const __bf16 *)(smem + (wave * 2 + buf) * A::v_bytes);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int cb = 0; cb < CB; ++cb)
                O[cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(value_fragment<D>(sV, 0, ks, cb, lane), pf[ks], O[cb], 0, 0, 0);
    }
    wait_loads<0>();

    merge_waves<D>(g, pl, it, row.live, O, m, s, smem, lane, wave, part_o, part_ms);
}

// ---- fp32 ----
// The same on v_mfma_f32_32x32x2_f32 (256 operations per CU and cycle, which bound it): a lane's chunks of a key row and a query
// row as in f32_tile.h; the second product takes the probabilities from the accumulators one element at a time, a
// contraction step over the keys of the two half-waves, and a value row's 32 channels per load straight from memory.  Beyond a few workgroups' latency
// the loads bound it: a block's page, keys and values are requested one after the other, none ahead (2 x 64 rows x 4 heads, 4096 keys, d = 128: products
// 7 of 49 us).
// The dots of 32 keys and 32 rows in four chains of D / 4 products: eight, as in f32_tile.h, leave no room beside the outputs (d = 128, 8
// sequences of one prefix of 2048 keys 26.3 us, so 21.6; 2 x 64 rows x 4 heads, 4096 keys 57.4, 49.5; d = 64 37.2, 29.0).
template <int D>
__device__ __forceinline__ f32x16 dots_f32(const f32x4 (&a)[D / 8], const float *sq) {
    f32x16 acc[4];
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[c][v] = 0.f;
#pragma unroll
    for (int i = 0; i < D / 8; ++i) {
        const f32x4 q = *(const f32x4 *)(sq + 8 * i);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i][e], q[e], acc[e], 0, 0, 0);
    }
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[0][v] = (acc[0][v] + acc[1][v]) + (acc[2][v] + acc[3][v]);
    return acc[0];
}
template <int D>
struct F32Attn {
    static constexpr int WAVES = 4, STEP = 32 * WAVES, LDQ = f32_ld(D);
    static constexpr size_t q_bytes = (size_t)32 * LDQ * 4, bytes = q_bytes > WaveMerge<D>::bytes ? q_bytes : WaveMerge<D>::bytes;
};
template <int D>
__global__ __launch_bounds__(256, 2) void shared_f32_kernel(SharedGeom g, SharedPlan pl, float *part_o, float2 *part_ms) {
    using A = F32Attn<D>;
    constexpr int CB = D / 32;
    __shared__ __attribute__((aligned(16))) char smem[A::bytes];
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
    {  // wave w: channels [w D / 4, + D / 4) of all rows, the half-waves alternate
        const float *p = (const float *)g.q + row.b * g.qs[0] + row.hq * g.qs[1] + row.t * g.qs[2];
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
            const int c = wave * (D / 4) + i * 8 + hf * 4;
            f32x4 x = *(const f32x4 *)(p + c);
            if (!row.live) x = f32x4{};
            *(f32x4 *)(sQ + col * A::LDQ + c) = x;
        }
    }
    __syncthreads();
    const float *sq = sQ + col * A::LDQ + 4 * hf;
    const float c_out = pl.c_out;
    const int limit = row.limit, limit_min = -reduce_lanes<1, 32>(-limit, OpMaxI{});
    f32x16 O[CB];
    float m = -INFINITY, s = 0.f;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int v = 0; v < 16; ++v) O[cb][v] = 0.f;
    for (int kb = it.begin + wave * 32; kb < it.end; kb += A::STEP) {
        const auto here = keys.at(kb + col, keys.entry(kb + col));
        const uint32_t there = (uint32_t)__builtin_amdgcn_ballot_w64(here.there);
        f32x4 a[D / 8];
#pragma unroll
        for (int i = 0; i < D / 8; ++i) a[i] = *(const f32x4 *)(here.k + 4 * hf + 8 * i);
        f32x16 acc = dots_f32<D>(a, sq);
        __builtin_amdgcn_sched_barrier(0);  // (value rows requested in front of the products take the registers of the chains)
        if (there != 0xffffffffu || kb + 31 > limit_min) {
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int at = 8 * (v >> 2) + 4 * hf + (v & 3);
                if (kb + at > limit || !((there >> at) & 1)) acc[v] = -INFINITY;
            }
        }
        float amax = -INFINITY;
#pragma unroll
        for (int v = 0; v < 16; ++v) amax = fmaxf(amax, acc[v]);
        amax = combine_lane_xor<32>(amax, OpMax{});
        const float mn = fmaxf(m, amax * c_out);
        const float mref = mn == -INFINITY ? 0.f : mn;
        const float corr = fast_exp2(m - mref);
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            acc[v] = fast_exp2(fmaf(acc[v], c_out, -mref));
            sum[v & 3] += acc[v];
        }
        s = s * corr + ((sum[0] + sum[1]) + (sum[2] + sum[3]));
        m = mn;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb)
#pragma unroll
            for (int v = 0; v < 16; ++v) O[cb][v] *= corr;
        const uint64_t mine = (uint64_t)(uintptr_t)here.v;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            const int from = 8 * (v >> 2) + 4 * hf + (v & 3);
            const uint32_t lo = __shfl((uint32_t)mine, from), hi = __shfl((uint32_t)(mine >> 32), from);
            const float *vr = (const float *)(((uint64_t)hi << 32) | lo) + col;
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) O[cb] = __builtin_amdgcn_mfma_f32_32x32x2f32(vr[cb * 32], acc[v], O[cb], 0, 0, 0);
        }
    }
    merge_waves<D>(g, pl, it, row.live, O, m, s, smem, lane, wave, part_o, part_ms);
}

// ---- joining a row's parts ----
// A thread takes four channels of a row and every SP-th part, four parts' loads in flight at once (bound by their latency: one
// after the other, 33 parts took 23 us); the SP threads of a channel meet in LDS.  Parts without a key have a reference of -inf and no
// output; rows without a prefix have no prefix parts.
struct JoinState {
    float m, s;
    f32x4 o;
    __device__ __forceinline__ void add(float m1, float s1, const f32x4 &o1) {
        const float mn = fmaxf(m, m1), ref = mn == -INFINITY ? 0.f : mn, f0 = exp2f(m - ref), f1 = exp2f(m1 - ref);
        s = s * f0 + s1 * f1;
        if (m1 != -INFINITY) {  // (else o1 may be anything)
#pragma unroll
            for (int c = 0; c < 4; ++c) o[c] = o[c] * f0 + o1[c] * f1;
        }
        m = mn;
    }
};
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
    T *out = (T *)g.out + b * g.os[0] + (h * g.G + gi) * g.os[1] + t * g.os[2] + ch;
    if constexpr (sizeof(T) == 2) {
        *(uint2 *)out = uint2{pack_bf16(x.o[0] * inv, x.o[1] * inv), pack_bf16(x.o[2] * inv, x.o[3] * inv)};
    } else {
        *(f32x4 *)out = f32x4{x.o[0] * inv, x.o[1] * inv, x.o[2] * inv, x.o[3] * inv};
    }
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
