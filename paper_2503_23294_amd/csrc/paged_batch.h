// What the calls on a page table share: which rows of a batch are whose, and where their tokens are.
#pragma once
#include "common.h"

namespace cocktail {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kMostPageSize = 65536;                    // tokens per page: a run's offsets stay below 2^24

// What kernels need to know of a batch: which rows are whose, and where their tokens are.
struct PagedBatch {
  char* pool;
  const int32_t* table;
  const int32_t* seq_lens;
  const int32_t* starts;    // or NULL: `uniform` rows for every sequence
  int32_t num_seqs, table_stride, page_size, num_pages;
  int32_t num_kv_heads;
  int32_t total, max_new, uniform;
};

// Rows [first, first + count) of sequence b; none where the range is not within the batch.
struct PagedSpan {
  int32_t first, count;
};
__device__ __forceinline__ PagedSpan paged_span(const PagedBatch& a, int b) {
  if (!a.starts) return {b * a.uniform, a.uniform};
  const int64_t s0 = a.starts[b], s1 = a.starts[b + 1];
  const bool ok = s0 >= 0 && s1 >= s0 && s1 <= a.total && s1 - s0 <= a.max_new;
  return {int32_t(s0), ok ? int32_t(s1 - s0) : 0};
}
// Tokens of a sequence, and those of them that its row of the table can hold (resize makes no more, but lengths may come from elsewhere).
__device__ __forceinline__ int paged_len(const PagedBatch& a, int b) {
  const int n = a.seq_lens[b];
  return n < 0 ? 0 : n;
}
__device__ __forceinline__ int paged_held(const PagedBatch& a, int len) {
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

int check_page_table(const cocktail_page_table* p);

}  // namespace cocktail
