// The 8-bit cache format: e4m3 codes, and for every 64 tokens of a segment and
// plane (KV head) one power of two 2^(e - 127), held as the byte e.  K and V
// have their own.  A code has 4 significant bits, so that a value of the cache
// is exact in bf16 and an attention over it is one over bf16 rows.
#pragma once

#include "common.hpp"

namespace rc {

constexpr int kBlk8 = 64;  // tokens per scale

// Scale blocks of a segment that starts at row `row` and is number `seg` of its
// cache: floor(row / 64) + seg, and as many after it as it has.  Segments do
// not share a slot, since floor(a / 64) + ceil(n / 64) <= floor((a + n) / 64) + 1,
// and rows / 64 + n_seg slots hold them all.
__host__ __device__ __forceinline__ long block_slot(long row, long seg) { return row / kBlk8 + seg; }
__host__ __device__ __forceinline__ long block_slots(long rows, long n_seg) { return rows / kBlk8 + n_seg; }

// 2^(e - 127); quantize writes 1 <= e <= 247.
__device__ __forceinline__ float block_scale(uint32_t e) { return __uint_as_float(e << 23); }

// Two codes of a dword (its low or high half), times scale (a power of two), as
// bf16: exact.
template <bool HI>
__device__ __forceinline__ uint32_t codes_to_bf16x2(uint32_t w, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HI));
}
// Eight codes.
__device__ __forceinline__ u32x4 codes_to_bf16x8(uint32_t lo, uint32_t hi, float scale) {
    return u32x4{codes_to_bf16x2<false>(lo, scale), codes_to_bf16x2<true>(lo, scale),
                 codes_to_bf16x2<false>(hi, scale), codes_to_bf16x2<true>(hi, scale)};
}

// Swizzle of the 16-byte chunks of K rows of codes in LDS: 16 consecutive rows of
// one chunk fall on distinct banks.
template <int HD>
__device__ __forceinline__ int k_mask8(int row) {
    return HD == 128 ? (row >> 1) & 7 : (row >> 2) & 3;
}

}  // namespace rc
