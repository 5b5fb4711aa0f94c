// The paged 4-bit cache (cocktail_fp4_*): page layout and codes.
#pragma once
#include "paged_batch.h"

namespace cocktail {

constexpr int kFp4Group = 32;                          // channels per scale
constexpr int kFp4LeastExp = -23, kFp4MostExp = 13;    // 0.5 * 2^-23 is the smallest fp16, 6 * 2^13 the largest that a code can be

// Bytes of one head's run in a page (K codes, V codes, K scales, V scales).
__host__ __device__ constexpr int64_t fp4_run_bytes(int head_dim, int page_size) {
  return int64_t(page_size) * (head_dim + head_dim / 16);
}

// Value in 0 .. 255 of byte k of a word, as the float 2^(value - 127).
__device__ __forceinline__ float fp4_scale(uint32_t word, int k) { return __builtin_bit_cast(float, ((word >> (8 * k)) & 255u) << 23); }

template <int BYTE>
__device__ __forceinline__ uint32_t fp4_pair(uint32_t codes, float scale) {
  return as_u32(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, BYTE));
}

int check_fp4_cache(const cocktail_fp4_cache* c);
// Arguments that store, gather and attention share; fills `a` on success.
int check_fp4_rows(const cocktail_fp4_cache* c, const void* x, const void* y, int32_t dtype, int64_t stride_t, int64_t stride_h,
                   int64_t total, const int32_t* starts, int heads, PagedBatch* a);

}  // namespace cocktail
