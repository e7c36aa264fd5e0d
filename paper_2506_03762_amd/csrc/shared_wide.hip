// Attention behind shared prefixes where many rows see the same keys: bf16, 65 rows and more (shared_attn.hip says what is computed,
// wide_tile.h how).
//
// 4 x 256 rows of 32 heads, 16384 keys: 373 us with all loads of a stage issued together and the largest logit taken in every block; 352 with
// the loads between the products; 311 with their addresses advanced in the vector ALU and a plain loop; now 304, 925 TFLOP/s with both launches
// (a library's product of 8192^3 reaches 1200): 1860 cycles for the 1024 of a block's products (the vector ALU 1000 of them, LDS reads 230, loads 90,
// the look at the sums 185), at 1.9 GHz, which the power leaves.  Products interleaved in other orders: no faster.
// 32 rows of 8 heads, 32768 keys: 49 of 71 us, of which 8 to the first products (25 MB that all workgroups request at once), 28 in the
// loop, 4 for the partial outputs.
#include <limits.h>

#include "shared_rows.h"
#include "wide_tile.h"

namespace aha {

template <int D, int RW>
__global__ __launch_bounds__(256, 1) void shared_wide_kernel(SharedGeom g, SharedPlan pl, float *part_o, float2 *part_ms) {
    using A = WideRows<D, RW>;
    constexpr int KS = D / 16, CB = D / 32;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), col = lane & 31, hf = lane >> 5;
    const int rw = wave % RW;
    SharedItem it;
    if (!shared_item(g, pl, (int)blockIdx.x, 64 * RW, A::KEYS, lane, it)) return;
    const int wrow = it.row0 + rw * 64;  // the wave's rows
    const bool mine = wrow < it.row1;
    if (it.begin >= it.end) {
        for (int i = tid; i < it.row1 - it.row0; i += 256)
            if (SharedRow(g, it, it.row0 + i).live) part_ms[partial_index(g, pl, it.h, it.part, it.row0 + i)] = make_float2(-INFINITY, 0.f);
        return;
    }
    const SharedKeys<__bf16> keys(g, it);
    int32_t *pages = (int32_t *)(smem + A::off_pages);
    const int entry0 = it.begin >> keys.shift;
    bool holes = false;  // in the item's pages (or so many pages that it is not known)
    if (!it.prefix) {
        const int all = ((it.end - 1) >> keys.shift) - entry0 + 1, n = min(A::kEntries, all);
        bool bad = n < all;
        for (int i = tid; i < n; i += 256) {
            const int page = keys.table[entry0 + i];
            pages[i] = page;
            bad |= page < 0 || page >= keys.pages;
        }
        holes = __syncthreads_or(bad);
    }
    auto entry = [&](int key) {  // the page of a tail's key (before `end`)
        const int i = (key >> keys.shift) - entry0;
        return i < A::kEntries ? pages[i] : keys.table[entry0 + i];
    };

    bf16x8 qf[2][KS];
    int limit[2], limit_min[2];
    uint32_t live[2];
    f32x16 O[2][CB];
    float m[2], s[2], sc[2];
    auto rows = [&] {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const SharedRow row(g, it, wrow + 32 * q + col);
            const __bf16 *p = (const __bf16 *)g.q + row.b * g.qs[0] + row.hq * g.qs[1] + row.t * g.qs[2] + hf * 8;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                qf[q][ks] = *(const bf16x8 *)(p + ks * 16);
                if (!row.live) qf[q][ks] = bf16x8{};
            }
            limit[q] = row.limit;
            live[q] = (uint32_t)__builtin_amdgcn_ballot_w64(row.live);
            limit_min[q] = uniform(-reduce_lanes<1, 32>(-limit[q], OpMaxI{}));
        }
    };
    wide_sweep<D, RW>(keys, it.prefix, holes, entry, smem, lane, wave, pl.c_out, qf, limit, limit_min, O, m, s, rows, [](auto) {},
                      [&] { return mine ? (it.end - it.begin + A::KEYS - 1) / A::KEYS : 0; });
    if (!wide_meet<D, RW>(O, m, s, sc, smem, lane, wave)) return;
    if (!mine) return;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        if (!((live[q] >> col) & 1)) continue;
        const int64_t p = partial_index(g, pl, it.h, it.part, wrow + 32 * q + col);
        if (hf == 0) part_ms[p] = make_float2(m[q], sc[q]);
#pragma unroll
        for (int cb = 0; cb < CB; ++cb)
#pragma unroll
            for (int v = 0; v < 16; v += 4)
                *(f32x4 *)(part_o + p * D + cb * 32 + 2 * v + 4 * hf) = f32x4{O[q][cb][v], O[q][cb][v + 1], O[q][cb][v + 2], O[q][cb][v + 3]};
    }
}

template <int D, int RW>
static hipError_t launch_wide_t(const SharedGeom &g, const SharedPlan &pl, float *part_o, float2 *part_ms, hipStream_t st) {
    using A = WideRows<D, RW>;
    static DeviceOnce once;
    const hipError_t e = device_once(once, [] {
        return hipFuncSetAttribute((const void *)shared_wide_kernel<D, RW>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)A::bytes);
    });
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((shared_wide_kernel<D, RW>), dim3((unsigned)(pl.prefix_items + pl.tail_items)), dim3(256), A::bytes, st, g, pl, part_o, part_ms);
    return hipGetLastError();
}

hipError_t launch_shared_wide(const SharedGeom &g, const SharedPlan &pl, int rows, float *part_o, float2 *part_ms, hipStream_t st) {
    if (g.d == 64) return rows == 128 ? launch_wide_t<64, 2>(g, pl, part_o, part_ms, st) : launch_wide_t<64, 4>(g, pl, part_o, part_ms, st);
    return rows == 128 ? launch_wide_t<128, 2>(g, pl, part_o, part_ms, st) : launch_wide_t<128, 4>(g, pl, part_o, part_ms, st);
}

}  // namespace aha
