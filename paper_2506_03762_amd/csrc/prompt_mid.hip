// Causal attention of packed prompts in tiles of four times 32 rows, bf16 (prompt_attn.hip says what is computed).
//
// A wave takes 32 rows of a query head; the four waves, heads of a group first, see nearly the same keys, whose rows and values' rows come to LDS once for
// all of them, 32 keys to a stage, straight from global memory.  Two workgroups share a CU, so that one multiplies while the other one starts, waits or
// writes its outputs, for which a tile of 256 rows (prompt_wide.hip) holds a CU for 10 us: 16 prompts of 200 tokens, 32 heads of 128 over 8, 24.5 us instead
// of 32, of 500 69 instead of 78, one of 1024 27 instead of 35.
//
// Bound by a tile's start and end, as far as the second workgroup does not hide them: 18432 tokens in equal prompts of 288 to 1536, 32 heads of 128 over 8, take
// 0.88 us per round of 512 tiles and block of 32 keys, which is what the matrix cores need (1.2 PFLOP/s), and 9.1 us per round besides (d = 64 0.57 and 3.7).
// So 24 prompts of up to 1500 tokens, 11.4 rounds, 257 us, spend 100 of them there (matrix cores 36 % busy, LDS instructions issue in 4 % of the
// waves' cycles).  Long prompts go to tiles of 256 rows, which read half as much from LDS per product: one of 16384 1935 us, here 2085 (matrix cores
// 49 % busy, so LDS at half of its rate; a third workgroup per CU, with three stages and no products ahead, 2331; stages of 64 keys 2223; keys and
// values in registers a phase ahead, as in wide_tile.h, 2081).
#include <type_traits>

#include "narrow_tile.h"
#include "prompt_tiles.h"
#include "wide_tile.h"

namespace aha {

// LDS: the stages, as in wide_tile.h; before the last two are requested their places hold the query rows of two waves each, in the end all of it
// the output rows (16 bytes further row by row: the halves of a row in other banks).
template <int D>
struct PromptMid {
    using A = WideRows<D, kUnits>;
    static constexpr int LD = D + 8, rows = KeyRows<D>::bytes(32), last_two = A::off_values + 2 * A::vbytes;
    static constexpr size_t bytes = last_two + (2 * rows > 2 * A::vbytes ? 2 * rows : 2 * A::vbytes);
    static_assert(A::kStages == 4 && A::KEYS == 32 && rows <= A::kbytes && 4 * 32 * LD * 2 <= bytes && bytes <= 80 * 1024, "half of a CU's LDS");
};

template <int D>
__global__ __launch_bounds__(256, 2) void prompt_mid_kernel(PromptGeom g) {
    using M = PromptMid<D>;
    using A = typename M::A;
    using R = KeyRows<D>;
    constexpr int KS = D / 16, CB = D / 32, S = A::kStages, NI = A::NI;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), col = lane & 31, hf = lane >> 5;
    PromptUnits it;
    if (!prompt_units<32>(g, g.item0 + (int)blockIdx.x, lane, it)) return;
    const int unit = it.first + wave, hq = it.h * g.G + unit % g.G, row0 = unit / g.G * 32;  // the wave's rows, counted from the prompt's start
    const int rows_here = max(0, min(32, it.n - row0));
    const __bf16 *kbase = (const __bf16 *)g.k + it.lo * g.ks[0] + it.h * g.ks[1], *vbase = (const __bf16 *)g.v + it.lo * g.vs[0] + it.h * g.vs[1];

    // ---- stages (places and permutations as in wide_tile.h) ----
    const uint32_t lds0 = uniform((int)(uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)smem);
    const int lr = lane / A::CPR, lc = lane % A::CPR;
    const int kchunk = lc ^ R::swizzle(lr), vchunk = lc ^ value_chunk_swizzle<D>(lr);
    auto load_to_lds = [&](const __bf16 *from, int to) {
        asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(from), "s"(uniform((int)lds0 + to)) : "memory");
    };
    const int64_t k_step = A::KEYS * g.ks[0], v_step = A::KEYS * g.vs[0];
    const __bf16 *k_at[NI], *v_at[NI];
    auto request = [&](int b) {  // (one after the other; past the last one: zeros)
        if (b > 0 && b < it.end / A::KEYS) {
#pragma unroll
            for (int j = 0; j < NI; ++j) k_at[j] += k_step, v_at[j] += v_step;
        } else {
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                const int key = b * A::KEYS + (wave + A::WAVES * j) * A::RPI + lr;
                k_at[j] = (key < it.end ? kbase + key * g.ks[0] : (const __bf16 *)kZeroRow) + kchunk * 8;
                v_at[j] = (key < it.end ? vbase + key * g.vs[0] : (const __bf16 *)kZeroRow) + vchunk * 8;
            }
        }
#pragma unroll
        for (int j = 0; j < NI; ++j) load_to_lds(k_at[j], b % S * A::kbytes + (wave + A::WAVES * j) * R::group);
#pragma unroll
        for (int j = 0; j < NI; ++j) load_to_lds(v_at[j], A::off_values + b % S * A::vbytes + (wave + A::WAVES * j) * 1024);
    };
    // this wave's loads but the last stage's have landed; behind the barrier so have all waves', and all waves are done with what they read
    auto barrier = [&](auto left) {
        __builtin_amdgcn_sched_barrier(0);
        wait_loads<decltype(left)::value>();
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    using OneStage = std::integral_constant<int, 2 * NI>;

    // ---- the wave's rows (behind the last one the prompt's last, whose results go nowhere) ----
    const int place = key_place<D>(lane);
    bf16x8 qf[KS];
    {
        const int at = (wave < 2 ? 2 * A::kbytes : M::last_two) + (wave & 1) * M::rows;
        const __bf16 *q = (const __bf16 *)g.q + hq * g.qs[1] + kchunk * 8;
#pragma unroll
        for (int j = 0; j < 32 / R::RPI; ++j) load_to_lds(q + (it.lo + min(row0 + j * R::RPI + lr, it.n - 1)) * g.qs[0], at + j * R::group);
        request(0);
        request(1);
        wait_loads<4 * NI>();
        asm volatile("" ::: "memory");
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) qf[ks] = key_fragment(smem + at, place, ks);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qf[ks]));
    }
    const int limit = min(row0 + col, it.n - 1), limit_min = uniform(min(row0, it.n - 1));
    f32x16 O[CB];
    float m, s;
    no_rows_yet(O, m, s);
    auto largest = [&](const f32x16 &x) {  // of a row's logits in a block, scaled
        float am[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int v = 0; v < 16; ++v) am[v & 1] = fmaxf(am[v & 1], x[v]);
        return combine_lane_xor<32>(fmaxf(am[0], am[1]), OpMax{}) * g.c_out;
    };
    auto products = [&](int b) {
        f32x16 x;
#pragma unroll
        for (int v = 0; v < 16; ++v) x[v] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
            x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(key_fragment(smem + b % S * A::kbytes, place, ks), qf[ks], x, 0, 0, 0);
        return x;
    };
    // Logits of block b that a row does not see become -inf; the reference is the largest logit of a row's first keys (wide_tile.h).
    auto finish = [&](f32x16 &acc, int b) {
        if (b * A::KEYS + A::KEYS - 1 > limit_min) {
            const int room = limit - b * A::KEYS - 4 * hf;
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[v] = 8 * (v >> 2) + (v & 3) > room ? -INFINITY : acc[v];
        }
        if (__builtin_amdgcn_ballot_w64(m == -INFINITY) != 0) {
            const float top = largest(acc);
            if (m == -INFINITY) m = top;
        }
    };
    const int stages = (it.end + A::KEYS - 1) / A::KEYS, blocks = uniform(rows_here > 0 ? (row0 + rows_here - 1) / A::KEYS + 1 : 0);
    barrier(OneStage{});  // stage 0 is here, the query rows have been read
    request(2);
    int st = 0;
    // Block st, whose logits are `acc`; those of the next one become `next`.  (Two blocks to a round of the loop: with
    // one, the logits are copied in each, and 16 prompts of 500 tokens take 71 us instead of 69.)
    auto step = [&](f32x16 &acc, f32x16 &next) {
        barrier(OneStage{});  // stage st + 1 is here, stage st - 1 done with
        request(st + 3);
        next = products(st + 1);  // beside this block's exponentials
        const float mref = m == -INFINITY ? 0.f : m;
        float sum[2] = {0.f, 0.f}, corr = 1.f;
        bf16x8 pf[2];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const float pr = fast_exp2(fmaf(acc[e], g.c_out, -mref));
            sum[e & 1] += pr;
            pf[e >> 3][e & 7] = (__bf16)pr;
        }
        const float all = sum[0] + sum[1];
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(all > kWideMost) != 0, 0)) {
            // far above the reference: a new one, the largest logit, and these weights again
            m = fmaxf(m, largest(acc));
            const float mn = m == -INFINITY ? 0.f : m;
            corr = fast_exp2(mref - mn);
            s *= corr;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float pr = fast_exp2(fmaf(acc[e], g.c_out, -mn));
                s += pr;
                pf[e >> 3][e & 7] = (__bf16)pr;
            }
        } else {
            s += all;
        }
        // (within that branch the compiler copies all outputs to other registers and back in every block: a prompt of 16384 2283 us)
        if (__builtin_amdgcn_ballot_w64(corr != 1.f) != 0) {
#pragma unroll
            for (int cb = 0; cb < CB; ++cb)
#pragma unroll
                for (int v = 0; v < 16; ++v) O[cb][v] *= corr;
        }
        const __bf16 *sV = (const __bf16 *)(smem + A::off_values + st % S * A::vbytes);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int cb = 0; cb < CB; ++cb)
                O[cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(value_fragment<D>(sV, 0, ks, cb, lane), pf[ks], O[cb], 0, 0, 0);
        if (++st < blocks) finish(next, st);
    };
    if (blocks > 0) {
        f32x16 x = products(0), y;
        finish(x, 0);
        while (true) {
            step(x, y);
            if (st >= blocks) break;
            step(y, x);
            if (st >= blocks) break;
        }
    }
    for (; st < stages; ++st) {  // (only its share of the loads)
        barrier(OneStage{});
        request(st + 3);
    }
    barrier(std::integral_constant<int, 0>{});  // (the last requests, past the range, write to LDS)

    // ---- the rows leave by way of LDS as whole ones ----
    constexpr int LD = M::LD, CPR = D / 8, RPI = 64 / CPR;
    __bf16 *rows_out = (__bf16 *)smem + wave * 32 * LD;
    const float sc = combine_lane_xor<32>(s, OpSum{}), f = 1.f / sc;
    if (hf == 0 && g.lse && col < rows_here) g.lse[(int64_t)hq * g.tokens + it.lo + row0 + col] = (m + log2f(sc)) * kLn2;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int v = 0; v < 16; v += 4)
            store_output(rows_out + col * LD + cb * 32 + 2 * v + 4 * hf, f32x4{O[cb][v], O[cb][v + 1], O[cb][v + 2], O[cb][v + 3]}, f);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __bf16 *out = (__bf16 *)g.out + (it.lo + row0) * g.os[0] + hq * g.os[1];
#pragma unroll
    for (int i = 0; i < 32 / RPI; ++i) {
        const int r = i * RPI + lane / CPR, c = lane % CPR * 8;
        const u32x4 x = *(const u32x4 *)(rows_out + r * LD + c);
        if (r < rows_here) *(u32x4 *)(out + r * g.os[0] + c) = x;
    }
}

template <int D>
static hipError_t launch_mid_t(const PromptGeom &g, const PromptPlan &pl, hipStream_t st) {
    static DeviceOnce once;
    const hipError_t e = device_once(once, [] {
        return hipFuncSetAttribute((const void *)prompt_mid_kernel<D>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)PromptMid<D>::bytes);
    });
    if (e != hipSuccess) return e;
    return launch_prompt_items(prompt_mid_kernel<D>, g, pl, PromptMid<D>::bytes, st);
}

hipError_t launch_prompt_mid(const PromptGeom &g, const PromptPlan &pl, hipStream_t st) {
    return g.d == 64 ? launch_mid_t<64>(g, pl, st) : launch_mid_t<128>(g, pl, st);
}

}  // namespace aha
