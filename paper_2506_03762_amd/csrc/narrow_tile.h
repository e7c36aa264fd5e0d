// One pass of a tile of 32 query rows over a range of keys: sum_j 2^(x_j - m) V_j, sum_j 2^(x_j - m) and m, x = c_out q . K_j.
//
// A workgroup's four waves take blocks of 32 keys in turn, each with all rows.  Keys (channels of the values) are on M, rows on N, so that the
// accumulator elements of a lane, its row's weights, are those that it supplies to the second product.  Every wave ends with results of
// its own, relative to a reference of its own, per row (lane % 32); sums over the two half-waves are left to the caller.
#pragma once

#include "f32_tile.h"
#include "key_places.h"
#include "value_rows.h"

namespace aha {

constexpr float kLn2 = 0.69314718055994531f;
constexpr float kRefSlack = 8.f;  // log2 units that a reference may lie below the running maximum

// bf16: keys go to registers, values to LDS, both a block ahead.
template <int D>
struct NarrowRows {
    static constexpr int WAVES = 4, STEP = 32 * WAVES, CPR = D / 8, RPI = 64 / CPR, NI = 32 / RPI;
    static constexpr size_t v_bytes = 32 * D * 2;   // a block's value rows
    static constexpr size_t stage_bytes = 2 * WAVES * v_bytes;
};
template <int CB>
__device__ __forceinline__ void no_rows_yet(f32x16 (&O)[CB], float &m, float &s) {
    m = -INFINITY;
    s = 0.f;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int v = 0; v < 16; ++v) O[cb][v] = 0.f;
}
// The weights of the 32 keys from kb on, by their products `acc`: rounded to bf16 in `pf`, added to s; reference and outputs moved where these exceed it.
template <int CB, class Block>
__device__ __forceinline__ void weigh_block(f32x16 &acc, int kb, uint32_t there, int limit, int limit_min, float c_out, int hf, float &m, float &s,
                                            f32x16 (&O)[CB], bf16x8 (&pf)[2], Block block) {
    if (there != 0xffffffffu || kb + 31 > limit_min) {
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            const int at = 8 * (v >> 2) + 4 * hf + (v & 3);
            if (kb + at > limit || !((there >> at) & 1)) acc[v] = -INFINITY;
        }
    }
    block(kb, acc);
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
}
// ONCE: the values are read past the caches, as no other tile reads them (64 caches of up to 4096 tokens, 8 x 4 heads of 128 channels 160 us, so 156; the
// keys too 191: a lane's pieces of a row come with eight loads, which then read it again).  `limit`: the last key that the lane's row sees.
// `block(kb, acc)` is told the products of the 32 keys from kb on, those that a row does not see -inf.
template <int D, bool ONCE = false, class Keys, class Block>
__device__ __forceinline__ void narrow_sweep(const Keys &keys, const bf16x8 (&qf)[D / 16], int limit, float c_out, char *smem, int lane, int wave,
                                             f32x16 (&O)[D / 32], float &m, float &s, Block block) {
    using A = NarrowRows<D>;
    constexpr int KS = D / 16, CB = D / 32;
    const int col = lane & 31, hf = lane >> 5, limit_min = -reduce_lanes<1, 32>(-limit, OpMaxI{});
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
            if constexpr (ONCE)
                asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off nt"
                             :
                             : "v"(src), "s"(lds0 + buf * (int)A::v_bytes + j * 1024)
                             : "memory");
            else
                asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
                             :
                             : "v"(src), "s"(lds0 + buf * (int)A::v_bytes + j * 1024)
                             : "memory");
        }
    };
    bf16x8 a[KS];
    auto load_keys = [&](const __bf16 *k) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) a[ks] = load_global<bf16x8>(k + hf * 8 + ks * 16);
    };

    int kb = keys.begin + wave * 32;
    int next_entry = keys.entry(kb + A::STEP + col);
    auto here = keys.at(kb + col, keys.entry(kb + col));
    request_values(here.v, 0);
    load_keys(here.k);
    for (int buf = 0; kb < keys.end; kb += A::STEP, buf ^= 1) {
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
        bf16x8 pf[2];
        weigh_block(acc, kb, there, limit, limit_min, c_out, hf, m, s, O, pf, block);
        const __bf16 *sV = (const __bf16 *)(smem + (wave * 2 + buf) * A::v_bytes);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int cb = 0; cb < CB; ++cb)
                O[cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(value_fragment<D>(sV, 0, ks, cb, lane), pf[ks], O[cb], 0, 0, 0);
    }
    wait_loads<0>();
}

// The same with the keys by way of LDS, too: whole rows, of which a lane's pieces straight from memory are a quarter of a line each, eight times.  Keys and
// values are read from there together, then the next block's are requested: a longer chain than above, but less for the L1, which all waves of a CU share.  d = 128, one
// prompt of 512 tokens, 32 heads over 8 15.9 us, so 13.6, of 2048, 8 over 2, 36.5, 29.9, of 4096, 2 heads 42.3, 40.5; d = 64, 9 of up to 777, 6 heads over 2, 13.5,
// 11.7, one of 4096, 2 heads, a workgroup per CU, 25.0, 28.3.  Caches in pages, whose rows' addresses come lane by lane: 64 of 1000 tokens 46, 53.
template <int D>
struct StagedRows {
    static constexpr int k_bytes = KeyRows<D>::bytes(32), bytes = k_bytes + 32 * D * 2;
    static constexpr size_t stage_bytes = 4 * bytes;
};
template <int D, class Keys>
__device__ __forceinline__ void staged_sweep(const Keys &keys, const bf16x8 (&qf)[D / 16], int limit, float c_out, char *smem, int lane, int wave,
                                             f32x16 (&O)[D / 32], float &m, float &s) {
    using A = NarrowRows<D>;
    using S = StagedRows<D>;
    using R = KeyRows<D>;
    constexpr int KS = D / 16, CB = D / 32;
    const int hf = lane >> 5, limit_min = -reduce_lanes<1, 32>(-limit, OpMaxI{});
    char *own = smem + wave * S::bytes;
    const uint32_t lds0 = uniform((int)((uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)own));
    const int lr = lane / A::CPR, kchunk = (lane % A::CPR) ^ R::swizzle(lr), vchunk = (lane % A::CPR) ^ value_chunk_swizzle<D>(lr);
    auto load_to_lds = [&](const __bf16 *from, int to) {
        asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(from), "s"(lds0 + to) : "memory");
    };
    auto request = [&](int kb) {
#pragma unroll
        for (int j = 0; j < A::NI; ++j) load_to_lds(keys.at(kb + j * A::RPI + lr, 0).k + kchunk * 8, j * R::group);
#pragma unroll
        for (int j = 0; j < A::NI; ++j) load_to_lds(keys.at(kb + j * A::RPI + lr, 0).v + vchunk * 8, S::k_bytes + j * 1024);
    };
    int kb = keys.begin + wave * 32;
    request(kb);
    const int place = key_place<D>(lane);
    const __bf16 *sV = (const __bf16 *)(own + S::k_bytes);
    for (; kb < keys.end; kb += A::STEP) {
        __builtin_amdgcn_sched_barrier(0);
        wait_loads<0>();
        asm volatile("" ::: "memory");
        bf16x8 a[KS], vf[2 * CB];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) a[ks] = key_fragment(own, place, ks);
#pragma unroll
        for (int i = 0; i < 2 * CB; ++i) vf[i] = value_fragment<D>(sV, 0, i / CB, i % CB, lane);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(a[ks]));
#pragma unroll
        for (int i = 0; i < 2 * CB; ++i) asm volatile("" : "+v"(vf[i]));
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        request(kb + A::STEP);
        f32x16 acc;
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[v] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[ks], qf[ks], acc, 0, 0, 0);
        bf16x8 pf[2];
        const int left = keys.end - kb;
        weigh_block(acc, kb, left >= 32 ? 0xffffffffu : (1u << left) - 1, limit, limit_min, c_out, hf, m, s, O, pf, [](int, const f32x16 &) {});
#pragma unroll
        for (int i = 0; i < 2 * CB; ++i) O[i % CB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[i], pf[i / CB], O[i % CB], 0, 0, 0);
    }
    wait_loads<0>();
}

// The dots of 32 keys and 32 rows in four chains of D / 4 products: eight, as in f32_tile.h, leave no room beside the outputs (d = 128, 8
// sequences of one prefix of 2048 keys 26.3 us, so 21.6; 2 x 64 rows x 4 heads, 4096 keys 57.4, 49.5, d = 64 37.2, 29.0, which are 28.9 and 21.1 with loads
// ahead).
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
// fp32: v_mfma_f32_32x32x2_f32 (256 operations per CU and cycle, which bound it beyond a few blocks' latency); a lane's chunks of a key row and a query
// row as in f32_tile.h (`sq`: its row in LDS, from its half's first chunk on);
// the second product takes the weights from the accumulators one element at a time, a contraction step over the keys of the
// two half-waves, and a value row's 32 channels per load straight from memory.  With nothing requested ahead a prompt of 512 tokens, 2 heads of 64, took
// 21.8 us, so 15.3.
template <int D, class Keys, class Block>
__device__ __forceinline__ void f32_sweep(const Keys &keys, const float *sq, int limit, float c_out, int lane, int wave, f32x16 (&O)[D / 32],
                                          float &m, float &s, Block block) {
    using A = NarrowRows<D>;
    constexpr int CB = D / 32;
    const int col = lane & 31, hf = lane >> 5, limit_min = -reduce_lanes<1, 32>(-limit, OpMaxI{});
    int kb = keys.begin + wave * 32;
    if (kb >= keys.end) return;
    // a block's values are requested in front of its dots, the next one's keys behind them, its page a block earlier
    int next_entry = keys.entry(kb + A::STEP + col);
    auto here = keys.at(kb + col, keys.entry(kb + col));
    f32x4 a[D / 8];
    auto load_keys = [&] {
#pragma unroll
        for (int i = 0; i < D / 8; ++i) a[i] = load_global<f32x4>(here.k + 4 * hf + 8 * i);
    };
    load_keys();
    for (; kb < keys.end; kb += A::STEP) {
        const uint32_t there = (uint32_t)__builtin_amdgcn_ballot_w64(here.there);
        float v_row[16][CB];
        const uint64_t mine = (uint64_t)(uintptr_t)here.v;
        auto load_values = [&](int v) {
            const int from = 8 * (v >> 2) + 4 * hf + (v & 3);
            const uint32_t lo = __shfl((uint32_t)mine, from), hi = __shfl((uint32_t)(mine >> 32), from);
            const float *vr = (const float *)(((uint64_t)hi << 32) | lo) + col;
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) v_row[v][cb] = load_global<float>(vr + cb * 32);
        };
        constexpr int AHEAD = D == 64 ? 16 : 0;  // (d = 128: they do not fit beside the dots' chains)
#pragma unroll
        for (int v = 0; v < AHEAD; ++v) load_values(v);
        here = keys.at(kb + A::STEP + col, next_entry);
        next_entry = keys.entry(kb + 2 * A::STEP + col);
        __builtin_amdgcn_sched_barrier(0);
        f32x16 acc = dots_f32<D>(a, sq);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int v = AHEAD; v < 16; ++v) load_values(v);
        load_keys();
        __builtin_amdgcn_sched_barrier(0);
        if (there != 0xffffffffu || kb + 31 > limit_min) {
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int at = 8 * (v >> 2) + 4 * hf + (v & 3);
                if (kb + at > limit || !((there >> at) & 1)) acc[v] = -INFINITY;
            }
        }
        block(kb, acc);
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
#pragma unroll
        for (int v = 0; v < 16; ++v)
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) O[cb] = __builtin_amdgcn_mfma_f32_32x32x2f32(v_row[v][cb], acc[v], O[cb], 0, 0, 0);
    }
}

// The waves' results meet.  Lane: row lane % 32, accumulator element v of channel block cb: channel 32 cb + 8 (v / 4) + 4 (lane / 32) + v % 4.
// Every wave scales its output to the largest reference, half of the channels at a time meet in LDS, and a thread adds four channels of the
// waves' rows (with a channel at a time and its weights formed there, 4 us of an item's 10; so 1).
//   row(M, sum)       lanes below 32 of the first wave, for their live row: reference and sum over all waves
//   store(q, ch, o)   four channels of live row q; sums[q] is its sum
template <int D>
struct WaveMerge {
    static constexpr int WAVES = 4, HC = D / 2, LDO = HC + 4;  // channels at a time, floats of a row
    static constexpr size_t o_bytes = (size_t)WAVES * 32 * LDO * 4, off_sums = o_bytes + (size_t)WAVES * 32 * 8, bytes = off_sums + 32 * 4;
};
template <int D, class Row, class Store>
__device__ __forceinline__ void meet_waves(int rows, bool live_row, f32x16 (&O)[D / 32], float m, float s, char *smem, int lane, int wave, Row row,
                                           Store store) {
    using A = WaveMerge<D>;
    constexpr int CB = D / 32, CPR = A::HC / 4;
    const int tid = wave * 64 + lane, col = lane & 31, hf = lane >> 5;
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
    if (tid < 32) ((float *)(smem + A::off_sums))[col] = all;
    if (tid < 32 && live_row) row(M, all);
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
            store(q, hc * A::HC + ch, o);
        }
    }
}

// LDS of a kernel of these sweeps: the values' blocks (fp32: the query rows), later the waves' results.
template <class T, int D, bool STAGED = false>
constexpr size_t narrow_lds() {
    const size_t swept = sizeof(T) == 4 ? (size_t)32 * f32_ld(D) * 4 : STAGED ? StagedRows<D>::stage_bytes : NarrowRows<D>::stage_bytes;
    return swept > WaveMerge<D>::bytes ? swept : WaveMerge<D>::bytes;
}
// Its workgroups per CU, at least.  Three where their LDS (32 KB each) and registers allow it without spills, bf16 with d = 64: there latency is what a
// block of keys mostly waits for (16 prompts of 200 tokens, 6 heads over 2: 9.3 us, with two 11.2; 64 caches of up to 4096 tokens, 8 x 4 heads 60.5 and 62.9;
// with four the registers spill).
template <class T, int D>
constexpr int kNarrowWorkgroups = sizeof(T) == 2 && D == 64 ? 3 : 2;
// Query row `q` of lane % 32 (its 16-byte fragments, or zeros) to the tile's rows in LDS, fp32: wave w takes channels [w D / 4, + D / 4) of all rows, the
// half-waves alternate.
template <int D>
__device__ __forceinline__ void stage_f32_rows(float *sq, const float *q, bool live, int lane, int wave) {
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
        const int c = wave * (D / 4) + i * 8 + (lane >> 5) * 4;
        f32x4 x = *(const f32x4 *)(q + c);
        if (!live) x = f32x4{};
        *(f32x4 *)(sq + (lane & 31) * f32_ld(D) + c) = x;
    }
}

// Four channels of an output row, rounded once.
template <class T>
__device__ __forceinline__ void store_output(T *to, const f32x4 &o, float f) {
    if constexpr (sizeof(T) == 2) *(uint2 *)to = uint2{pack_bf16(o[0] * f, o[1] * f), pack_bf16(o[2] * f, o[3] * f)};
    else *(f32x4 *)to = f32x4{o[0] * f, o[1] * f, o[2] * f, o[3] * f};
}

// Parts of a row, joined one after the other.
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

}  // namespace aha
