// cocktail_fp4_store / cocktail_fp4_gather: 16-bit rows into the pages of the 4-bit cache and back.  Bound by memory: 4 D bytes of K and V
// a token and kv head on the one side, 17/16 D on the other.
#include <hip/hip_runtime.h>

#include "fp4_common.h"

namespace cocktail {

// A thread's share is eight channels of a quad of tokens (four consecutive ones from a multiple of four: a V piece holds them side by
// side, and no two threads write the same byte): sixteen bytes of each of four rows, so that neighbouring threads read and write
// neighbouring memory on both sides.  The four threads of a group of 32 channels find its scale together.  (A whole group per
// thread, 64 bytes of a row, was 4 times slower on the way back, whose stores then leave lines half written, and a third slower on
// the way in.)  Measured: 32K tokens of 32 heads of 128, 0.68 GB each way, stored in 133 us (5.1 TB/s) and read back in 97 (7.0); a step
// of 8 sequences 4 us each way.
// Numbering: per quad (K or V, head, eight channels), channels fastest.  Quads are numbered over the batch with room for one that
// starts and one that ends inside a sequence's range: those of sequence b are first[b] / 4 + 2 b and following.
struct Fp4Item {
  int seq, pos, row, lo, hi;   // sequence, position of the quad's first token, row of that token; tokens lo .. hi-1 of the quad are in the range
  int head, part, is_v;        // part: channels 8 part .. 8 part + 7
  bool active;
};

__device__ __forceinline__ int quad_number(int first, int b) { return (first >> 2) + 2 * b; }

// starts[0 .. num_seqs] in LDS; the thread's item from its number in the grid.
template <int HD>
__device__ __forceinline__ Fp4Item find_item(const Fp4Batch& a, const int32_t* lds_starts) {
  constexpr int kParts = HD / 8;
  Fp4Item it;
  const uint32_t per_quad = 2u * kParts * a.num_kv_heads;
  const uint64_t begin = uint64_t(blockIdx.x) * 256;
  const uint64_t quad0 = begin / per_quad;                      // (of the workgroup: scalar)
  uint32_t unit = uint32_t(begin - quad0 * per_quad) + threadIdx.x;
  const uint32_t ahead = unit / per_quad;
  const int quad = int(quad0 + ahead);
  unit -= ahead * per_quad;
  it.part = unit % kParts;
  unit /= kParts;
  it.is_v = unit >= uint32_t(a.num_kv_heads);
  it.head = it.is_v ? unit - a.num_kv_heads : unit;
  // the last sequence whose first quad is not behind this one
  int b = 0, e = a.num_seqs;
  while (e - b > 1) {
    const int m = (b + e) >> 1;
    if (quad_number(lds_starts[m], m) <= quad) b = m;
    else e = m;
  }
  it.seq = b;
  const Fp4Span s = fp4_span(a, b);
  const int p0 = fp4_len(a, b) - s.count;                            // position of the range's first token (the last one's is below 2^31)
  const int q0 = p0 >> 2;                                            // its quad (rounded down: p0 may be negative)
  const int k = quad - quad_number(lds_starts[b], b);
  it.active = k >= 0 && s.count > 0 && q0 + k <= (p0 + s.count - 1) >> 2;
  if (!it.active) return it;
  it.pos = (q0 + k) * 4;
  it.row = s.first + (it.pos - p0);
  it.lo = p0 > it.pos ? p0 - it.pos : 0;
  const int left = p0 + s.count - it.pos;
  it.hi = left < 4 ? left : 4;
  return it;
}

__device__ __forceinline__ void load_starts(const Fp4Batch& a, int32_t* lds) {
  // a range that is no range is cut to the batch, so that the numbers ascend as far as they can; fp4_span leaves it out
  for (int b = threadIdx.x; b <= a.num_seqs; b += 256) {
    const int v = a.starts ? a.starts[b] : b * a.uniform;
    lds[b] = v < 0 ? 0 : v > a.total ? a.total : v;
  }
  __syncthreads();
}

// The page's bytes for the item's head, or NULL.
__device__ __forceinline__ char* page_run(const Fp4Batch& a, const Fp4Item& it, int64_t run) {
  if (it.pos < 0) return nullptr;
  const int col = it.pos / a.page_size;
  if (col >= a.table_stride) return nullptr;
  const int page = a.table[int64_t(it.seq) * a.table_stride + col];
  if (uint32_t(page) >= uint32_t(a.num_pages)) return nullptr;
  return a.pool + (int64_t(page) * a.num_kv_heads + it.head) * run;
}

__device__ __forceinline__ uint32_t pk_max_u16(uint32_t x, uint32_t y) {
  typedef uint16_t us2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(us2, x), __builtin_bit_cast(us2, y)));
}

template <bool BF16, int BYTE>
__device__ __forceinline__ uint32_t encode_pair(uint32_t old, uint32_t x, float scale) {
  if constexpr (BF16) {
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(old, __builtin_bit_cast(b2, x), scale, BYTE);
  } else {
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(old, as_h2(x), scale, BYTE);
  }
}

// The value of the lane of the same four that differs in the bits of X (1, 2).
template <int X>
__device__ __forceinline__ uint32_t of_quad_lane(uint32_t v) {
  return uint32_t(__builtin_amdgcn_update_dpp(0, int(v), X == 1 ? 0xB1 : 0x4E, 0xF, 0xF, true));
}

// Four words of each of four lanes: word i of lane j becomes word j of lane i.
__device__ __forceinline__ u32x4 transpose_quad(u32x4 v, int j) {
  // swap the off-diagonal blocks of two, then of one
  const bool hi = j & 2, odd = j & 1;
  const uint32_t a = of_quad_lane<2>(hi ? v[0] : v[2]), b = of_quad_lane<2>(hi ? v[1] : v[3]);
  if (hi) v[0] = a, v[1] = b;
  else v[2] = a, v[3] = b;
  const uint32_t c = of_quad_lane<1>(odd ? v[0] : v[1]), d = of_quad_lane<1>(odd ? v[2] : v[3]);
  if (odd) v[0] = c, v[2] = d;
  else v[1] = c, v[3] = d;
  return v;
}

// Eight channels in 16 bits, a quarter of a group whose other quarters the lanes of the same four have -> their codes, and the scale byte.
// The conversion instruction divides by the power of two and rounds to nearest even, which is the definition; it would make a NaN
// the largest code, so those are cleared before (their bits, taken as an integer without the sign, are the only ones above infinity's).
template <bool BF16>
__device__ __forceinline__ uint32_t encode_part(u32x4 x, uint32_t* scale_byte) {
  constexpr uint32_t kInf = BF16 ? 0x7f80u : 0x7c00u;
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) m = pk_max_u16(m, x[i] & 0x7fff7fffu);
  uint32_t top = (m & 0xffffu) > (m >> 16) ? m & 0xffffu : m >> 16;
  if (top > kInf) {
    top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t w = x[i];
      if ((w & 0x7fffu) > kInf) w &= 0xffff0000u;
      if (((w >> 16) & 0x7fffu) > kInf) w &= 0xffffu;
      x[i] = w;
      const uint32_t lo = w & 0x7fffu, hi = (w >> 16) & 0x7fffu;
      top = lo > top ? lo : top;
      top = hi > top ? hi : top;
    }
  }
  uint32_t other = of_quad_lane<1>(top);
  top = other > top ? other : top;
  other = of_quad_lane<2>(top);
  top = other > top ? other : top;
  float f;
  if constexpr (BF16) f = __builtin_bit_cast(float, top << 16);
  else f = float(__builtin_bit_cast(_Float16, uint16_t(top)));
  int e = int(__builtin_bit_cast(uint32_t, f) >> 23) - 2;   // biased; below the least one for zeros and subnormals
  e = e < kFp4LeastExp + 127 ? kFp4LeastExp + 127 : e > kFp4MostExp + 127 ? kFp4MostExp + 127 : e;
  *scale_byte = uint32_t(e);
  const float scale = __builtin_bit_cast(float, uint32_t(e) << 23);
  uint32_t w = 0;
  w = encode_pair<BF16, 0>(w, x[0], scale);
  w = encode_pair<BF16, 1>(w, x[1], scale);
  w = encode_pair<BF16, 2>(w, x[2], scale);
  return encode_pair<BF16, 3>(w, x[3], scale);
}

struct Fp4Rows {
  char* k;
  char* v;
  int64_t stride_t, stride_h;   // bytes
  const int32_t* status;
};

template <int HD, bool BF16>
__global__ __launch_bounds__(256) void fp4_store_kernel(Fp4Batch a, Fp4Rows r) {
  extern __shared__ int32_t lds_starts[];
  load_starts(a, lds_starts);
  if (r.status[0] != 0) return;   // there was no room for these tokens
  const Fp4Item it = find_item<HD>(a, lds_starts);
  if (!it.active) return;
  const int64_t run = fp4_run_bytes(HD, a.page_size);
  char* base = page_run(a, it, run);
  if (!base) return;
  const char* src = (it.is_v ? r.v : r.k) + it.head * r.stride_h + it.part * 16;
  u32x4 x[4] = {};
#pragma unroll
  for (int t = 0; t < 4; ++t)
    if (t >= it.lo && t < it.hi) x[t] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + (it.row + t) * r.stride_t));
  const int at = it.pos % a.page_size, p = a.page_size;
  u32x4 codes;
  uint32_t scale[4];
#pragma unroll
  for (int t = 0; t < 4; ++t) codes[t] = encode_part<BF16>(x[t], &scale[t]);
  const int j = it.part & 3, group = it.part >> 2;
  if (!it.is_v) {
    // lane j of the four writes token j: sixteen bytes of its row
    const u32x4 row = transpose_quad(codes, j);
    if (j >= it.lo && j < it.hi) {
      *reinterpret_cast<u32x4*>(base + (at + j) * (HD / 2) + group * 16) = row;
      base[p * HD + (at + j) * (HD / 32) + group] = char(j == 0 ? scale[0] : j == 1 ? scale[1] : j == 2 ? scale[2] : scale[3]);
    }
    return;
  }
  char* dst = base + p * (HD / 2) + (at / 4) * (2 * HD) + it.part * 16;
  char* sc = base + p * HD + p * (HD / 32) + (at / 4) * (HD / 8) + group * 4;
  if (it.lo == 0 && it.hi == 4) {
    *reinterpret_cast<u32x4*>(dst) = codes;
    if (j == 0) *reinterpret_cast<uint32_t*>(sc) = scale[0] | scale[1] << 8 | scale[2] << 16 | scale[3] << 24;
    return;
  }
#pragma unroll
  for (int t = 0; t < 4; ++t)
    if (t >= it.lo && t < it.hi) {
      *reinterpret_cast<uint32_t*>(dst + t * 4) = codes[t];
      if (j == 0) sc[t] = char(scale[t]);
    }
}

template <bool BF16>
__device__ __forceinline__ uint32_t decode_word(uint32_t codes, float scale, int byte) {
  switch (byte) {
    case 0: return BF16 ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0)) : fp4_pair<0>(codes, scale);
    case 1: return BF16 ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1)) : fp4_pair<1>(codes, scale);
    case 2: return BF16 ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2)) : fp4_pair<2>(codes, scale);
    default: return BF16 ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3)) : fp4_pair<3>(codes, scale);
  }
}

// Codes that are read once.  Past the caches where the runs begin at their lines, so that a wave reads whole ones (32K tokens, 32 heads, stored
// and read back: 268 -> 225 us); a line that two waves share would be fetched twice (64 channels, pages of 16: 67 -> 90 us).
template <bool LINES>
__device__ __forceinline__ u32x4 load_codes(const char* p) {
  const u32x4* x = reinterpret_cast<const u32x4*>(p);
  if constexpr (LINES) return __builtin_nontemporal_load(x);
  else return *x;
}

template <int HD, bool BF16, bool LINES>
__global__ __launch_bounds__(256) void fp4_gather_kernel(Fp4Batch a, Fp4Rows r) {
  extern __shared__ int32_t lds_starts[];
  load_starts(a, lds_starts);
  const Fp4Item it = find_item<HD>(a, lds_starts);
  if (!it.active) return;
  const int64_t run = fp4_run_bytes(HD, a.page_size);
  const char* base = page_run(a, it, run);
  const int j = it.part & 3, group = it.part >> 2;
  u32x4 codes = {};                 // of the thread's channels, by token
  uint32_t scales = 0x7f7f7f7fu;
  if (base) {
    const int at = it.pos % a.page_size, p = a.page_size;
    if (!it.is_v) {
      const u32x4 row = load_codes<LINES>(base + (at + j) * (HD / 2) + group * 16);   // of token j
      codes = transpose_quad(row, j);
      const uint8_t* sc = reinterpret_cast<const uint8_t*>(base + p * HD + at * (HD / 32) + group);
      scales = sc[0] | sc[HD / 32] << 8 | sc[2 * (HD / 32)] << 16 | uint32_t(sc[3 * (HD / 32)]) << 24;
    } else {
      codes = load_codes<LINES>(base + p * (HD / 2) + (at / 4) * (2 * HD) + it.part * 16);
      scales = *reinterpret_cast<const uint32_t*>(base + p * HD + p * (HD / 32) + (at / 4) * (HD / 8) + group * 4);
    }
  }
  char* dst = (it.is_v ? r.v : r.k) + it.head * r.stride_h + it.part * 16;
#pragma unroll
  for (int t = 0; t < 4; ++t)
    if (t >= it.lo && t < it.hi) {
      const float s = fp4_scale(scales, t);
      const u32x4 x = {decode_word<BF16>(codes[t], s, 0), decode_word<BF16>(codes[t], s, 1), decode_word<BF16>(codes[t], s, 2), decode_word<BF16>(codes[t], s, 3)};
      __builtin_nontemporal_store(x, reinterpret_cast<u32x4*>(dst + (it.row + t) * r.stride_t));
    }
}

int check_fp4_cache(const cocktail_fp4_cache* c) {
  if (!c) return fail(COCKTAIL_EINVAL, "cache is NULL");
  if (int rc = check_page_table(&c->pages)) return rc;
  if (c->num_kv_heads < 1 || c->num_kv_heads > 1024) return fail(COCKTAIL_EINVAL, "num_kv_heads %d is not in 1 .. 1024", c->num_kv_heads);
  if (c->head_dim != 64 && c->head_dim != 128)
    return fail(COCKTAIL_EUNSUPPORTED, "kernels are built for head_dim 64 and 128, got %d", c->head_dim);
  if (c->pages.page_size % 16 || c->pages.page_size > kFp4MostPage)
    return fail(COCKTAIL_EINVAL, "page_size %d is not a multiple of 16 up to %d", c->pages.page_size, kFp4MostPage);
  // (positions and the numbers of keys a little behind the last one are ints)
  if (int64_t(c->pages.table_stride) * c->pages.page_size > (int64_t(1) << 31) - 256)
    return fail(COCKTAIL_EINVAL, "table_stride * page_size must be at most 2^31 - 256 for the cache");
  if (!c->pool) return fail(COCKTAIL_EINVAL, "pool is NULL");
  if (reinterpret_cast<uintptr_t>(c->pool) & 15) return fail(COCKTAIL_EALIGN, "pool must be 16-byte aligned");
  return COCKTAIL_OK;
}

int check_fp4_rows(const cocktail_fp4_cache* c, const void* x, const void* y, int32_t dtype, int64_t stride_t, int64_t stride_h,
                   int64_t total, const int32_t* starts, int heads, Fp4Batch* a) {
  if (int rc = check_fp4_cache(c)) return rc;
  if (dtype != COCKTAIL_FP16 && dtype != COCKTAIL_BF16) return fail(COCKTAIL_EINVAL, "dtype %d is neither COCKTAIL_FP16 nor COCKTAIL_BF16", dtype);
  if (total < 0 || total > (int64_t(1) << 30)) return fail(COCKTAIL_EINVAL, "total %lld is not in 0 .. 2^30", (long long)total);
  if (total && (!x || !y)) return fail(COCKTAIL_EINVAL, "the rows must not be NULL");
  if ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(y)) & 15) return fail(COCKTAIL_EALIGN, "the rows must be 16-byte aligned");
  if (stride_t < 0 || stride_h < 0 || stride_t % 8 || stride_h % 8 || stride_t > (int64_t(1) << 31) || stride_h > (int64_t(1) << 31))
    return fail(COCKTAIL_EINVAL, "strides must be multiples of 8 in 0 .. 2^31");
  if (heads > 1 && stride_h < c->head_dim) return fail(COCKTAIL_EINVAL, "heads overlap: stride_h %lld", (long long)stride_h);
  if (total > 1 && stride_t < c->head_dim) return fail(COCKTAIL_EINVAL, "rows overlap: stride_t %lld", (long long)stride_t);
  if (reinterpret_cast<uintptr_t>(starts) & 3) return fail(COCKTAIL_EALIGN, "starts must be 4-byte aligned");
  if (!starts && total % c->pages.num_seqs)
    return fail(COCKTAIL_EINVAL, "without starts the rows (%lld) must be a multiple of the sequences (%d)", (long long)total, c->pages.num_seqs);
  const cocktail_page_table& p = c->pages;
  *a = {static_cast<char*>(c->pool), p.table, p.seq_lens, starts, p.num_seqs, p.table_stride, p.page_size, p.num_pages, c->num_kv_heads,
        int32_t(total), int32_t(total), int32_t(total / p.num_seqs)};
  return COCKTAIL_OK;
}

}  // namespace cocktail

using namespace cocktail;

namespace {

template <class Kernel>
int launch_rows(Kernel kernel, const Fp4Batch& a, const Fp4Rows& r, int head_dim, void* stream, const char* what) {
  if (!a.total) return COCKTAIL_OK;
  const uint64_t quads = uint64_t(a.total) / 4 + 2 * uint64_t(a.num_seqs) + 1;
  const uint64_t blocks = (quads * (2 * a.num_kv_heads * (head_dim / 8)) + 255) / 256;
  if (blocks >= uint64_t(1) << 24) return fail(COCKTAIL_EINVAL, "%s of %d rows of %d heads is more than one launch takes", what, a.total, a.num_kv_heads);
  const hipError_t e = launch_lds(kernel, dim3(uint32_t(blocks)), dim3(256), (a.num_seqs + 1) * sizeof(int32_t), static_cast<hipStream_t>(stream), a, r);
  if (e != hipSuccess) return fail(COCKTAIL_EHIP, "%s launch failed: %s", what, hipGetErrorString(e));
  return COCKTAIL_OK;
}

}  // namespace

extern "C" int cocktail_fp4_page_bytes(int32_t num_kv_heads, int32_t head_dim, int32_t page_size, int64_t* bytes) {
  if (!bytes) return fail(COCKTAIL_EINVAL, "bytes is NULL");
  if (num_kv_heads < 1 || num_kv_heads > 1024) return fail(COCKTAIL_EINVAL, "num_kv_heads %d is not in 1 .. 1024", num_kv_heads);
  if (head_dim != 64 && head_dim != 128) return fail(COCKTAIL_EUNSUPPORTED, "kernels are built for head_dim 64 and 128, got %d", head_dim);
  if (page_size < 16 || page_size % 16 || page_size > kFp4MostPage)
    return fail(COCKTAIL_EINVAL, "page_size %d is not a multiple of 16 up to %d", page_size, kFp4MostPage);
  *bytes = num_kv_heads * fp4_run_bytes(head_dim, page_size);
  return COCKTAIL_OK;
}

extern "C" int cocktail_fp4_store(const cocktail_fp4_cache* cache, const void* k, const void* v, int32_t dtype, int64_t stride_t,
                                  int64_t stride_h, int64_t total, const int32_t* starts, void* stream) {
  Fp4Batch a;
  if (int rc = check_fp4_rows(cache, k, v, dtype, stride_t, stride_h, total, starts, cache ? cache->num_kv_heads : 0, &a)) return rc;
  const Fp4Rows r = {static_cast<char*>(const_cast<void*>(k)), static_cast<char*>(const_cast<void*>(v)), 2 * stride_t, 2 * stride_h, cache->pages.status};
  const bool d128 = cache->head_dim == 128;
  if (dtype == COCKTAIL_BF16)
    return launch_rows(d128 ? fp4_store_kernel<128, true> : fp4_store_kernel<64, true>, a, r, cache->head_dim, stream, "store");
  return launch_rows(d128 ? fp4_store_kernel<128, false> : fp4_store_kernel<64, false>, a, r, cache->head_dim, stream, "store");
}

extern "C" int cocktail_fp4_gather(const cocktail_fp4_cache* cache, void* k, void* v, int32_t dtype, int64_t stride_t, int64_t stride_h,
                                   int64_t total, const int32_t* starts, void* stream) {
  Fp4Batch a;
  if (int rc = check_fp4_rows(cache, k, v, dtype, stride_t, stride_h, total, starts, cache ? cache->num_kv_heads : 0, &a)) return rc;
  const Fp4Rows r = {static_cast<char*>(k), static_cast<char*>(v), 2 * stride_t, 2 * stride_h, nullptr};
  typedef void (*Kernel)(Fp4Batch, Fp4Rows);
  static const Kernel kernels[2][2][2] = {   // head_dim, dtype, whole lines
      {{fp4_gather_kernel<64, false, false>, fp4_gather_kernel<64, false, true>}, {fp4_gather_kernel<64, true, false>, fp4_gather_kernel<64, true, true>}},
      {{fp4_gather_kernel<128, false, false>, fp4_gather_kernel<128, false, true>}, {fp4_gather_kernel<128, true, false>, fp4_gather_kernel<128, true, true>}}};
  const bool lines = fp4_run_bytes(cache->head_dim, cache->pages.page_size) % 128 == 0 && reinterpret_cast<uintptr_t>(cache->pool) % 128 == 0;
  return launch_rows(kernels[cache->head_dim == 128][dtype == COCKTAIL_BF16][lines], a, r, cache->head_dim, stream, "gather");
}
