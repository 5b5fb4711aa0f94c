// The paged 4-bit cache (cocktail_fp4_*): page layout, and how a batch's rows find their sequence.
#pragma once
#include "common.h"

namespace cocktail {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kFp4Group = 32;                          // channels per scale
constexpr int kFp4LeastExp = -23, kFp4MostExp = 13;    // 0.5 * 2^-23 is the smallest fp16, 6 * 2^13 the largest that a code can be

constexpr int kFp4MostPage = 65536;                    // tokens per page: a run's offsets stay below 2^24

// Bytes of one head's run in a page (K codes, V codes, K scales, V scales).
__host__ __device__ constexpr int64_t fp4_run_bytes(int head_dim, int page_size) {
  return int64_t(page_size) * (head_dim + head_dim / 16);
}

// What kernels need to know of a batch: which rows are whose, and where their tokens are.
struct Fp4Batch {
  char* pool;
  const int32_t* table;
  const int32_t* seq_lens;
  const int32_t* starts;    // or NULL: `uniform` rows for every sequence
  int32_t num_seqs, table_stride, page_size, num_pages;
  int32_t num_kv_heads;
  int32_t total, max_new, uniform;
};

// Rows [first, first + count) of sequence b; none where the range is not within the batch.
struct Fp4Span {
  int32_t first, count;
};
__device__ __forceinline__ Fp4Span fp4_span(const Fp4Batch& a, int b) {
  if (!a.starts) return {b * a.uniform, a.uniform};
  const int64_t s0 = a.starts[b], s1 = a.starts[b + 1];
  const bool ok = s0 >= 0 && s1 >= s0 && s1 <= a.total && s1 - s0 <= a.max_new;
  return {int32_t(s0), ok ? int32_t(s1 - s0) : 0};
}
// Tokens of a sequence, and those of them that its row of the table can hold (resize makes no more, but lengths may come from elsewhere).
__device__ __forceinline__ int fp4_len(const Fp4Batch& a, int b) {
  const int n = a.seq_lens[b];
  return n < 0 ? 0 : n;
}
__device__ __forceinline__ int fp4_held(const Fp4Batch& a, int len) {
  const int most = a.table_stride * a.page_size;
  return len > most ? most : len;
}

// Inclusive prefix sum over the lanes of a wave, without a trip through shared memory: shifts inside rows of 16, then the last lane of a row
// to the rows behind it.
__device__ __forceinline__ int wave_prefix(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
  return x;
}

// Value in 0 .. 255 of byte k of a word, as the float 2^(value - 127).
__device__ __forceinline__ float fp4_scale(uint32_t word, int k) { return __builtin_bit_cast(float, ((word >> (8 * k)) & 255u) << 23); }

template <int BYTE>
__device__ __forceinline__ uint32_t fp4_pair(uint32_t codes, float scale) {
  return as_u32(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, BYTE));
}

int check_page_table(const cocktail_page_table* p);
int check_fp4_cache(const cocktail_fp4_cache* c);
// Arguments that store, gather and attention share; fills `a` on success.
int check_fp4_rows(const cocktail_fp4_cache* c, const void* x, const void* y, int32_t dtype, int64_t stride_t, int64_t stride_h,
                   int64_t total, const int32_t* starts, int heads, Fp4Batch* a);

}  // namespace cocktail
