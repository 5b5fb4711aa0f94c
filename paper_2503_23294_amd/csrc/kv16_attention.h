// What the kernels of cocktail_kv16_attention share.
#pragma once
#include "kv16_common.h"
#include "paged_attention.h"

namespace cocktail {

typedef __bf16 b8 __attribute__((ext_vector_type(8)));

// A call as the kernels of the 16-bit cache see it: batch.pool is K's.
struct Kv16Attention {
  PagedAttention p;
  const char* v_pool;
};

// 16x16x32 products of either type; operands are handed around as words.
template <bool BF16>
__device__ __forceinline__ f32x4 product16(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (BF16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
}
template <bool BF16>
__device__ __forceinline__ uint32_t pack_weights(float lo, float hi) {
  return pack_out(lo, hi, BF16);
}
// Eight ones.
template <bool BF16>
__device__ __forceinline__ u32x4 ones16() {
  constexpr uint32_t kOne = BF16 ? 0x3f803f80u : 0x3c003c00u;
  return u32x4{kOne, kOne, kOne, kOne};
}

}  // namespace cocktail
