// Value rows in LDS as the attention kernels keep them: brought there straight from global memory, read as fragments of V^T.
#pragma once

#include "score_tile.h"

namespace aha {

// The wave's value rows in LDS: row-major without padding (direct loads from global memory
// place the 64 lanes' 16-byte chunks back to back), the 16-byte chunks of row R permuted by
// XOR with swz(R), so that the four rows of a transposing read fall into different banks.
template <int D>
__device__ __forceinline__ int value_chunk_swizzle(int row) {
    return (4 * (row & 3)) % (D / 8);
}

// s_waitcnt vmcnt(N) alone (the other counters at their maxima): bits 3:0 and 15:14 hold
// vmcnt, 6:4 expcnt, 11:8 lgkmcnt.
template <int N>
__device__ __forceinline__ void wait_loads() {
    __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (15 << 8) | ((N >> 4) << 14));
}

// A fragment of V^T for channel block cb, key block mb, contraction step ks: this lane's
// channel cb * 32 + lane % 32 of the eight keys that its accumulator elements 8 ks .. 8 ks + 7
// of key block mb stand for (rows mb * 32 + 16 ks + 8 (e / 4) + e % 4 + 4 (lane / 32)): two
// runs of four consecutive keys, eight rows apart.  A lane wants a COLUMN of four elements at
// a time: ds_read_b64_tr_b16 reads, per group of 16 lanes, a tile of 4 rows x 16 elements -
// lane s of the group supplies the address of row s / 4, elements 4 (s % 4) .. + 3 - and hands
// lane j of the group column j of that tile.  Two such reads make a fragment, with no
// repacking in the vector ALU.
template <int D>
__device__ __forceinline__ bf16x8 value_fragment(const __bf16 *sV, int mb, int ks, int cb,
                                                 int lane) {
    using lds_ptr = s16x4 __attribute__((address_space(3))) *;
    const int row = mb * 32 + 16 * ks + 4 * (lane >> 5) + ((lane >> 2) & 3);
    const int chunk = cb * 4 + ((lane & 16) >> 3) + ((lane & 3) >> 1);  // of elements 4 (s % 4) .. + 3
    // (rows 8 apart have the same swizzle)
    const __bf16 *p = sV + row * D + (chunk ^ value_chunk_swizzle<D>(row)) * 8 + 4 * (lane & 1);
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)p);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p + 8 * D));
    bf16x8 f;
    __builtin_memcpy(&f, &lo, 8);
    __builtin_memcpy((char *)&f + 8, &hi, 8);
    return f;
}

}  // namespace aha
