// One pass of a tile of 256 query rows (RW = 4) or 128 (RW = 2) over a range of keys, bf16: sum_j 2^(x_j - m) V_j, sum_j 2^(x_j - m) and m,
// x = c_out q . K_j.
//
// Bound by the matrix core and what keeps it waiting.  A wave owns two blocks of 32 rows, a workgroup's four waves 256 rows (RW = 4),
// or 128 whose keys two pairs of waves divide (RW = 2).  The keys' and values' rows come to LDS for all waves at once, 32 keys (RW = 2: 64) to
// a stage, kStages deep, straight from global memory.  Per 32 keys a wave runs two phases, and in each the matrix core
// multiplies for one row block while the vector ALU forms the exponentials of the other:
//
//   phase 0 of keys i:  S1(i) = K(i) Q1, O1 += V(i-1) P1(i-1)   beside   P0(i) = 2^(S0(i) - m0)
//   phase 1 of keys i:  S0(i+1) = K(i+1) Q0, O0 += V(i) P0(i)   beside   P1(i) = 2^(S1(i) - m1)
//
// so that one wave per SIMD keeps both busy; a second one would not fit its registers (two outputs of 64, queries 64, keys 32,
// values 32, logits 32, probabilities 16, rounded to bf16).  A key or value fragment is read from LDS once for both row blocks, right behind its
// last use, and waits in registers for 16 products: half of the reads of a wave with one row block, for which
// LDS is as busy as the matrix core.
#pragma once

#include <limits.h>

#include "key_places.h"
#include "key_stages.h"
#include "value_rows.h"

namespace aha {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// A row's reference is the largest logit of its first keys, and stays until a block's weights add up to more than this: fp32
// and bf16 (which have the same exponents) hold them as exactly at that size as at 1.  So a block takes no maximum and,
// but for rows whose logits keep rising, no rescaling.
constexpr float kWideMost = 0x1p20f;

// x *= f where x lives in accumulator registers: written in assembly so that the compiler keeps it there on both ways past this
// rarely taken branch (else it copies all outputs to vector registers and back in every block).  The waits are those between a
// product and a read of its result, and between a write and a product.
template <int CB>
__device__ __forceinline__ void scale_outputs(f32x16 (&O)[CB], float f) {
    asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            float x = O[cb][v], y;
            asm volatile("v_accvgpr_read_b32 %1, %0\n\ts_nop 1\n\tv_mul_f32 %1, %1, %2\n\ts_nop 1\n\tv_accvgpr_write_b32 %0, %1\n\ts_nop 3"
                         : "+a"(x), "=&v"(y)
                         : "v"(f));
            O[cb][v] = x;
        }
    asm volatile("s_nop 15" ::: "memory");
}

template <int D, int RW>
struct WideRows {
    static constexpr int WAVES = 4, KW = WAVES / RW, KEYS = 32 * KW;
    static constexpr int CPR = D / 8, RPI = 64 / CPR, NI = KEYS / RPI / WAVES;  // load instructions per wave for a stage's keys (values)
    static constexpr int kStages = 4;  // (32 x 32768 keys, eight stages of 32 keys 75.8 us, four 72.7)
    static constexpr int kbytes = KeyRows<D>::bytes(KEYS), vbytes = KEYS * D * 2;
    static constexpr int off_values = kStages * kbytes, off_pages = off_values + kStages * vbytes;
    static constexpr int kEntries = 2048;  // page numbers kept in LDS (a longer range reads the others from memory)
    static constexpr size_t bytes = off_pages + kEntries * 4;
    static_assert(bytes <= 160 * 1024 && KEYS % (RPI * WAVES) == 0, "one CU's LDS, whole instructions per wave");
};

// The sweep.  `in_a_row`: the keys lie token by token, else in pages: entry(key) is the page of a key before the end, `holes`: one of them may be
// none.  `rows()` requests the wave's query rows and says the last key that each row sees and the least of these of either block;
// `take(n)`, n loads later, has them in the fragments qf.  `mine()`: blocks of 32 keys that the wave's rows see (0: it has no rows).  O, m and s are the
// wave's, s per half-wave.
template <int D, int RW, class Entry, class Rows, class Take, class Mine>
__device__ __forceinline__ void wide_sweep(const KeyPlaces<__bf16> &keys, bool in_a_row, bool holes, Entry entry, char *smem, int lane, int wave,
                                           float c_out, bf16x8 (&qf)[2][D / 16], int (&limit)[2], int (&limit_min)[2], f32x16 (&O)[2][D / 32],
                                           float (&m)[2], float (&s)[2], Rows rows, Take take, Mine mine) {
    using A = WideRows<D, RW>;
    constexpr int KS = D / 16, CB = D / 32, NV = 2 * CB, S = A::kStages, NI = A::NI, SLOTS = KS + NV, EL = 16 / SLOTS;
    const int col = lane & 31, hf = lane >> 5, kw = wave / RW;
    // ---- stages ----
    // Load j of a stage covers RPI rows of group wave + 4 j, lane -> row lane / CPR, place lane % CPR; the 16-byte chunks of a
    // row are permuted on the way.  The loads are assembly and the waits for them by hand (value_rows.h).
    const uint32_t lds0 = uniform((int)(uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)smem);
    const int lr = lane / A::CPR, lc = lane % A::CPR;
    const int kchunk = lc ^ KeyRows<D>::swizzle(lr), vchunk = lc ^ value_chunk_swizzle<D>(lr);
    const int stages = (keys.end - keys.begin + A::KEYS - 1) / A::KEYS;
    const int whole = in_a_row ? (keys.end - keys.begin) / A::KEYS : 0;  // stages whose rows follow from those of the one before
    const int64_t k_step = A::KEYS * keys.ks, v_step = A::KEYS * keys.vs;
    const __bf16 *k_at[NI], *v_at[NI];  // what the lane loads of the stage to come
    auto locate = [&](int stage) {      // (stages have to be located one by one; past the last one: zeros)
        if (stage > 0 && stage < whole) {
#pragma unroll
            for (int j = 0; j < NI; ++j) k_at[j] += k_step, v_at[j] += v_step;
            return;
        }
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            const int key = keys.begin + stage * A::KEYS + (wave + A::WAVES * j) * A::RPI + lr;
            const auto row = keys.at(key, !in_a_row && key < keys.end ? entry(key) : 0);
            k_at[j] = row.k + kchunk * 8;
            v_at[j] = row.v + vchunk * 8;
        }
    };
    auto load_to_lds = [&](const __bf16 *from, int to) {
        asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(from), "s"(uniform((int)lds0 + to)) : "memory");
    };
    auto request_keys = [&](int place, int j) { load_to_lds(k_at[j], place * A::kbytes + (wave + A::WAVES * j) * KeyRows<D>::group); };
    auto request_values = [&](int place, int j) {
        load_to_lds(v_at[j], A::off_values + place * A::vbytes + (wave + A::WAVES * j) * 1024);
    };
    auto request = [&](int stage) {
        locate(stage);
#pragma unroll
        for (int j = 0; j < NI; ++j) request_keys(stage % S, j);
#pragma unroll
        for (int j = 0; j < NI; ++j) request_values(stage % S, j);
    };

    // ---- the wave's rows, which travel with the first stages ----
    rows();
    // (a loop that is not unrolled, here and where it does not count: straight code that runs once is fetched from memory line by line)
#pragma unroll 1
    for (int i = 0; i < S - 1; ++i) request(i);
    take(std::integral_constant<int, 2 * NI * (S - 1)>{});
#pragma unroll
    for (int q = 0; q < 2; ++q)  // (no load of the compiler's is waited for in the loop)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qf[q][ks]));

    f32x16 acc[2];
    bf16x8 kf[KS], vf[NV], pf[2][2];
    m[0] = m[1] = -INFINITY;
    s[0] = s[1] = 0.f;
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
        for (int cb = 0; cb < CB; ++cb)
#pragma unroll
            for (int v = 0; v < 16; ++v) O[q][cb][v] = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) vf[i] = bf16x8{};
    pf[1][0] = pf[1][1] = bf16x8{};

    const int place = key_place<D>(lane);
    auto largest = [&](const f32x16 &x) {  // of a row's logits in a block, scaled
        float am[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int v = 0; v < 16; ++v) am[v & 1] = fmaxf(am[v & 1], x[v]);
        return combine_lane_xor<32>(fmaxf(am[0], am[1]), OpMax{}) * c_out;
    };
    // block b of the wave, in stage b: keys [key_of(b), + 32)
    auto key_of = [&](int b) { return keys.begin + b * A::KEYS + kw * 32; };
    auto key_rows = [&](int b) { return smem + b % S * A::kbytes + kw * KeyRows<D>::bytes(32); };
    auto value_rows = [&](int b) { return (const __bf16 *)(smem + A::off_values + b % S * A::vbytes) + kw * 32 * D; };
    // Logits of block b that row block q does not see become -inf; a row that has seen no key so far takes its reference, the
    // largest logit of its first keys.
    auto finish = [&](int q, int b) {
        const int kb = key_of(b);
        uint32_t there = 0xffffffffu;
        if (!in_a_row) {
            const int key = kb + col, page = key < keys.end ? entry(key) : -1;
            there = (uint32_t)__builtin_amdgcn_ballot_w64(page >= 0 && page < keys.pages);
        }
        if (kb + 32 > keys.end || kb + 31 > limit_min[q] || there != 0xffffffffu) {
            const int room = min(limit[q], keys.end - 1) - kb - 4 * hf;
            if (there == 0xffffffffu) {
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[q][v] = 8 * (v >> 2) + (v & 3) > room ? -INFINITY : acc[q][v];
            } else {
                there >>= 4 * hf;
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const int at = 8 * (v >> 2) + (v & 3);
                    if (at > room || !((there >> at) & 1)) acc[q][v] = -INFINITY;
                }
            }
        }
        if (__builtin_amdgcn_ballot_w64(m[q] == -INFINITY) != 0) {
            const float top = largest(acc[q]);
            if (m[q] == -INFINITY) m[q] = top;
        }
    };
    // A phase of block b: exponentials of row block q, products of the other one; in phase 0 the fragments are replaced by those of
    // the next keys and of these keys' values.  The vector work lies between the products in the order in which it is written (without
    // the empty assembly the compiler moves it behind them), and so do half of a later stage's loads: issued together they
    // hold the waves up, 16 cycles per load and wave.
    auto phase = [&](auto which, int b) {
        constexpr int q = decltype(which)::value, o = 1 - q;
        const char *next_keys = key_rows(b + 1);
        const __bf16 *these_values = value_rows(b);
        auto load = [&](int slot) {
            if (slot % (SLOTS / NI) != 0) return;
            if (q == 0) request_keys((b + S - 1) % S, slot / (SLOTS / NI));
            else request_values((b + S - 1) % S, slot / (SLOTS / NI));
        };
        float sum[2], pr[16];
        const float mref = m[q] == -INFINITY ? 0.f : m[q];
        auto pack = [&](int e) {  // e, e + 1
            bf16x2 two = {(__bf16)pr[e], (__bf16)pr[e + 1]};
            asm volatile("" : "+v"(two));
            pf[q][e >> 3][e & 7] = two[0];
            pf[q][e >> 3][(e & 7) + 1] = two[1];
        };
        auto weigh = [&](int slot) {  // (what uses an exponential comes one or two later: it takes its time)
#pragma unroll
            for (int e = EL * slot; e < EL * (slot + 1); ++e) {
                pr[e] = fast_exp2(fmaf(acc[q][e], c_out, -mref));
                keep_here(pr[e]);
                if (e == 1 || e == 2) sum[e - 1] = pr[e - 1];
                if (e > 2) sum[(e - 1) & 1] += pr[e - 1];
                if (e > 1) keep_here(sum[(e - 1) & 1]);
                if (e > 1 && !(e & 1)) pack(e - 2);
            }
        };
        const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            acc[o] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[ks], qf[o][ks], ks ? acc[o] : zero, 0, 0, 0);
            if (q == 0) kf[ks] = key_fragment(next_keys, place, ks);
            weigh(ks);
            load(ks);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            O[o][i % CB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[i], pf[o][i / CB], O[o][i % CB], 0, 0, 0);
            if (q == 0) vf[i] = value_fragment<D>(these_values, 0, i / CB, i % CB, lane);
            weigh(KS + i);
            load(KS + i);
            __builtin_amdgcn_sched_barrier(0);
        }
        pack(14);
        const float all = sum[0] + (sum[1] + pr[15]), before = s[q];
        s[q] += all;
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(all > kWideMost) != 0, 0)) {
            // far above the reference: a new one, the largest logit, and these weights again
            m[q] = fmaxf(m[q], largest(acc[q]));
            const float mn = m[q] == -INFINITY ? 0.f : m[q], corr = fast_exp2(mref - mn);
            s[q] = before * corr;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                pr[e] = fast_exp2(fmaf(acc[q][e], c_out, -mn));
                s[q] += pr[e];
            }
#pragma unroll
            for (int e = 0; e < 16; e += 2) pack(e);
            scale_outputs(O[q], corr);
        }
    };
    // this wave's loads of the next stage have landed (those of the S - 3 behind it may be in flight); behind the barrier so have
    // all waves', and all waves are done with the stage before this one, whose place the next request takes
    auto advance = [&] {
        __builtin_amdgcn_sched_barrier(0);
        wait_loads<2 * NI * (S - 3)>();
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    advance();
    const int blocks = uniform(mine());
    if (blocks > 0) {
        const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) kf[ks] = key_fragment(key_rows(0), place, ks);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) acc[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[ks], qf[0][ks], ks ? acc[0] : zero, 0, 0, 0);
        finish(0, 0);
        // (one hole in an item sends all its blocks the long way: 4 x 256 rows of 32 heads, tails of 8192 alone 155 us without holes, 182
        // with one in each tail)
        const int plain = holes ? 0 : (int)max((int64_t)0, min((int64_t)keys.end, (int64_t)min(limit_min[0], limit_min[1]) + 1) - keys.begin) / A::KEYS;
        using P0 = std::integral_constant<int, 0>;
        using P1 = std::integral_constant<int, 1>;
        for (int st = 0; st < blocks;) {
            advance();
            locate(st + S - 1);
            phase(P0{}, st);
            finish(1, st);
            phase(P1{}, st);
            if (++st < blocks) finish(0, st);
            // where all rows see all keys, and the next ones, and have a reference, there are only the phases
            if (__builtin_amdgcn_ballot_w64(m[0] == -INFINITY || m[1] == -INFINITY) != 0) continue;
            for (; st + 2 <= plain; ++st) {
                advance();
                locate(st + S - 1);
                phase(P0{}, st);
                phase(P1{}, st);
            }
        }
    }
    for (int st = blocks; st < stages; ++st) {  // (only its share of the loads)
        advance();
        request(st + S - 1);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) O[1][i % CB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[i], pf[1][i / CB], O[1][i % CB], 0, 0, 0);
    wait_loads<0>();  // (the last requests, past the range, write to LDS)

}

// The results of the second pair of waves go to the first one's (RW = 2), which then have all of their rows; sums over the half-waves, too.
// false: the wave has given its results away.
template <int D, int RW>
__device__ __forceinline__ bool wide_meet(f32x16 (&O)[2][D / 32], float (&m)[2], const float (&s)[2], float (&sc)[2], char *smem, int lane, int wave) {
    constexpr int CB = D / 32, KW = WideRows<D, RW>::KW;
    const int rw = wave % RW, kw = wave / RW;
#pragma unroll
    for (int q = 0; q < 2; ++q) sc[q] = combine_lane_xor<32>(s[q], OpSum{});
    if constexpr (KW == 2) {  // the second pair's results go to the first one's through LDS
        __syncthreads();
        float *sO = (float *)smem + (size_t)rw * 2 * CB * 16 * 64;
        float2 *sMS = (float2 *)((float *)smem + (size_t)RW * 2 * CB * 16 * 64) + rw * 2 * 64;
        if (kw == 1) {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                sMS[q * 64 + lane] = make_float2(m[q], sc[q]);
#pragma unroll
                for (int cb = 0; cb < CB; ++cb)
#pragma unroll
                    for (int v = 0; v < 16; v += 4)
                        *(f32x4 *)(sO + (((q * CB + cb) * 4 + v / 4) * 64 + lane) * 4) =
                            f32x4{O[q][cb][v], O[q][cb][v + 1], O[q][cb][v + 2], O[q][cb][v + 3]};
            }
        }
        __syncthreads();
        if (kw == 1) return false;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const float2 ms = sMS[q * 64 + lane];
            const float M = fmaxf(m[q], ms.x), mref = M == -INFINITY ? 0.f : M;
            const float f0 = fast_exp2(m[q] - mref), f1 = fast_exp2(ms.x - mref);
            sc[q] = sc[q] * f0 + ms.y * f1;
            m[q] = M;
#pragma unroll
            for (int cb = 0; cb < CB; ++cb)
#pragma unroll
                for (int v = 0; v < 16; v += 4) {
                    const f32x4 x = *(const f32x4 *)(sO + (((q * CB + cb) * 4 + v / 4) * 64 + lane) * 4);
#pragma unroll
                    for (int c = 0; c < 4; ++c) O[q][cb][v + c] = O[q][cb][v + c] * f0 + x[c] * f1;
                }
        }
    }
    return true;
}

}  // namespace aha
