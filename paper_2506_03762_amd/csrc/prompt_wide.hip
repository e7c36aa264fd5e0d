// Causal attention of packed prompts in tiles of four times 64 rows, bf16 (prompt_attn.hip says what is computed, wide_tile.h how).
//
// A wave takes 64 rows of a query head and leaves out the keys behind its last one.  One prompt of 16384 tokens, 32 heads of 128 over 8: 1935 us, 1.13
// PFLOP/s, as a library's product of 8192^3 reaches 1.16: power bounds both.  A tile's start, the blocks with masks and its outputs take 10 us, so
// that shorter prompts go to tiles of 128 rows; a workgroup that takes several tiles one after the other, its next keys and rows requested during the last
// blocks, gained nothing (1930).
#include "narrow_tile.h"
#include "prompt_tiles.h"
#include "wide_tile.h"

namespace aha {

// LDS: the stages, then for every wave its query rows, later its output rows (16 bytes further row by row: the halves of a row in other banks).
template <int D>
struct PromptWide {
    static constexpr int LD = D + 8;
    static constexpr size_t rows = KeyRows<D>::bytes(64) > 64 * LD * 2 ? KeyRows<D>::bytes(64) : 64 * LD * 2, off_rows = WideRows<D, kUnits>::bytes,
                            bytes = off_rows + 4 * rows;
    static_assert(rows % 16 == 0 && off_rows % 1024 == 0 && bytes <= 160 * 1024, "one CU's LDS");
};

template <int D>
__global__ __launch_bounds__(256, 1) void prompt_wide_kernel(PromptGeom g) {
    using A = WideRows<D, kUnits>;
    constexpr int KS = D / 16, CB = D / 32;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), col = lane & 31, hf = lane >> 5;
    PromptUnits it;
    if (!prompt_units<64>(g, g.item0 + (int)blockIdx.x, lane, it)) return;
    const int unit = it.first + wave, hq = it.h * g.G + unit % g.G, row0 = unit / g.G * 64;  // the wave's rows, counted from the prompt's start
    const int rows_here = max(0, min(64, it.n - row0));
    KeyPlaces<__bf16> keys;
    keys.in_a_row((const __bf16 *)g.k + it.lo * g.ks[0] + it.h * g.ks[1], (const __bf16 *)g.v + it.lo * g.vs[0] + it.h * g.vs[1], g.ks[0], g.vs[0]);
    keys.begin = 0;
    keys.end = it.end;
    bf16x8 qf[2][KS];
    int limit[2], limit_min[2];
    f32x16 O[2][CB];
    float m[2], s[2], sc[2];
    // A load covers RPI whole rows (of fragments, 32 rows' 32 bytes at a time, they took 3 us); behind the last row the prompt's last one, whose
    // results go nowhere.
    char *own_rows = smem + PromptWide<D>::off_rows + wave * PromptWide<D>::rows;
    auto rows = [&] {
        using R = KeyRows<D>;
        const uint32_t to = uniform((int)(uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)own_rows);
        const int lr = lane / R::CPR, chunk = (lane % R::CPR) ^ R::swizzle(lr);
        const __bf16 *q = (const __bf16 *)g.q + hq * g.qs[1] + chunk * 8;
#pragma unroll 4
        for (int j = 0; j < 64 / R::RPI; ++j) {
            const __bf16 *from = q + (it.lo + min(row0 + j * R::RPI + lr, it.n - 1)) * g.qs[0];
            asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(from), "s"(to + j * R::group) : "memory");
        }
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            limit[q] = min(row0 + 32 * q + col, it.n - 1);
            limit_min[q] = uniform(min(row0 + 32 * q, it.n - 1));
        }
    };
    auto take = [&](auto later) {
        wait_loads<decltype(later)::value>();
        asm volatile("" ::: "memory");
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) qf[q][ks] = key_fragment(own_rows + q * KeyRows<D>::bytes(32), key_place<D>(lane), ks);
    };
    // blocks that begin at or before the wave's last row
    auto blocks = [&] {
        return rows_here > 0 ? (row0 + rows_here - 1) / A::KEYS + 1 : 0;
    };
    wide_sweep<D, kUnits>(keys, true, false, [](int) { return 0; }, smem, lane, wave, g.c_out, qf, limit, limit_min, O, m, s, rows, take,
                      blocks);
    if (!wide_meet<D, kUnits>(O, m, s, sc, smem, lane, wave)) return;
    // The rows leave by way of LDS as whole ones, too.
    constexpr int LD = PromptWide<D>::LD, CPR = D / 8, RPI = 64 / CPR;
    __bf16 *rows_out = (__bf16 *)own_rows;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const float f = 1.f / sc[q];
        if (hf == 0 && g.lse && 32 * q + col < rows_here)
            g.lse[(int64_t)hq * g.tokens + it.lo + row0 + 32 * q + col] = (m[q] + log2f(sc[q])) * kLn2;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb)
#pragma unroll
            for (int v = 0; v < 16; v += 4)
                store_output(rows_out + (32 * q + col) * LD + cb * 32 + 2 * v + 4 * hf, f32x4{O[q][cb][v], O[q][cb][v + 1], O[q][cb][v + 2], O[q][cb][v + 3]},
                             f);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __bf16 *out = (__bf16 *)g.out + (it.lo + row0) * g.os[0] + hq * g.os[1];
#pragma unroll
    for (int i = 0; i < 64 / RPI; ++i) {
        const int r = i * RPI + lane / CPR, c = lane % CPR * 8;
        const u32x4 x = *(const u32x4 *)(rows_out + r * LD + c);
        if (r < rows_here) *(u32x4 *)(out + r * g.os[0] + c) = x;
    }
}

template <int D>
static hipError_t launch_wide_t(const PromptGeom &g, const PromptPlan &pl, hipStream_t st) {
    static DeviceOnce once;
    const hipError_t e = device_once(once, [] {
        return hipFuncSetAttribute((const void *)prompt_wide_kernel<D>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)PromptWide<D>::bytes);
    });
    if (e != hipSuccess) return e;
    return launch_prompt_items(prompt_wide_kernel<D>, g, pl, PromptWide<D>::bytes, st);
}

hipError_t launch_prompt_wide(const PromptGeom &g, const PromptPlan &pl, hipStream_t st) {
    return g.d == 64 ? launch_wide_t<64>(g, pl, st) : launch_wide_t<128>(g, pl, st);
}

}  // namespace aha
