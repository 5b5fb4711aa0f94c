// cocktail_kv16_append: new tokens into 16-bit pages, K and the queries rotated by their position on the way.
#include <hip/hip_runtime.h>

#include <cmath>

#include "kv16_common.h"

namespace cocktail {

struct Kv16Rows {
  const char *k, *v, *q;
  char *k_pool, *v_pool, *q_out;
  int64_t stride_t, stride_h, q_stride_t, q_stride_h;   // bytes
  const int32_t *positions, *status;
  const double* inv_freq;
  int32_t rotary, interleaved, q_heads;
  float factor;
};

template <bool BF16>
__device__ __forceinline__ float low_of(uint32_t w) {
  if constexpr (BF16) return __builtin_bit_cast(float, w << 16);
  else return float(__builtin_bit_cast(_Float16, uint16_t(w)));
}
template <bool BF16>
__device__ __forceinline__ float high_of(uint32_t w) {
  if constexpr (BF16) return __builtin_bit_cast(float, w & 0xffff0000u);
  else return float(__builtin_bit_cast(_Float16, uint16_t(w >> 16)));
}
template <bool BF16>
__device__ __forceinline__ uint32_t pack_pair(float lo, float hi) {
  if constexpr (BF16) {
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, b2{__bf16(lo), __bf16(hi)});
  } else {
    return as_u32(h2{_Float16(lo), _Float16(hi)});
  }
}

// What the threads of a workgroup have to know of a token.
struct Kv16Token {
  int64_t place;   // first byte of the token in the run of kv head 0, or -1: not stored
  int32_t pos;     // for the rotation
  int32_t valid;   // the row belongs to a sequence
};

// Bound by memory: 4 D bytes a head in and out; 32K tokens of 32 + 8 + 8 heads of 128 (805 MB) 154 us, 5.2 TB/s, where a copy of as much reaches 5.0 .. 5.4;
// a step of 8 tokens is a launch and a chain of four loads, 4.2 us.
// A workgroup takes TOKENS rows (blockIdx.x) and a part of their heads (blockIdx.y), a thread sixteen channels of a head at a time: two pieces of
// sixteen bytes that are the two halves of eight pairs (or eight neighbouring pairs), or are only moved.  What a token needs is found out
// once, and the sines and cosines are one per (token, pair) in LDS for all heads.
template <int HD, bool BF16, int TOKENS>
__global__ __launch_bounds__(256) void kv16_append_kernel(PagedBatch a, Kv16Rows r) {
  constexpr int kParts = HD / 16;   // units of sixteen channels per head
  extern __shared__ int32_t lds_starts[];
  __shared__ Kv16Token tokens[TOKENS];
  __shared__ float turn_cos[TOKENS][HD / 2], turn_sin[TOKENS][HD / 2];
  const int tid = threadIdx.x;
  const int t0 = int(blockIdx.x) * TOKENS;
  if (a.starts) {
    // a range that is no range is cut to the batch; paged_span leaves it out
    for (int b = tid; b <= a.num_seqs; b += 256) {
      const int v = a.starts[b];
      lds_starts[b] = v < 0 ? 0 : v > a.total ? a.total : v;
    }
    __syncthreads();
  }
  if (tid < TOKENS) {
    const int t = t0 + tid;
    Kv16Token x = {-1, 0, 0};
    if (t < a.total) {
      int b = 0;
      if (!a.starts) {
        b = t / a.uniform;
      } else {
        // the last sequence that does not start behind the row (those before it with the same start are empty)
        int e = a.num_seqs;
        while (e - b > 1) {
          const int m = (b + e) >> 1;
          if (lds_starts[m] <= t) b = m;
          else e = m;
        }
      }
      const PagedSpan s = paged_span(a, b);
      if (t >= s.first && t < s.first + s.count) {
        const int pos = paged_len(a, b) - s.count + (t - s.first);   // (negative where the sequence is shorter than its range)
        x.valid = 1;
        x.pos = r.positions ? r.positions[t] : pos;
        const int col = pos < 0 ? -1 : pos / a.page_size;
        if (col >= 0 && col < a.table_stride && r.status[0] == 0) {
          const int page = a.table[int64_t(b) * a.table_stride + col];
          if (uint32_t(page) < uint32_t(a.num_pages)) x.place = (int64_t(page) * a.num_kv_heads * a.page_size + (pos - col * a.page_size)) * (2 * HD);
        }
      }
    }
    tokens[tid] = x;
  }
  __syncthreads();
  const int pairs = r.rotary / 2;
  for (int i = tid; i < TOKENS * pairs; i += 256) {
    const int t = i / pairs, pair = i - t * pairs;
    // the angle in turns, with what its products were rounded by; whole turns are dropped before it becomes binary32
    constexpr double kTurn = 0.15915494309189535, kTurnRest = -9.839338337591243e-18;   // 1 / (2 pi) to 106 bits
    const double pos = tokens[t].pos, freq = r.inv_freq[pair];
    const double per = freq * kTurn, per_rest = fma(freq, kTurn, -per) + freq * kTurnRest;
    const double turns = pos * per, rest = fma(pos, per, -turns) + pos * per_rest;
    float s, c;
    sincospif(float(2.0 * ((turns - rint(turns)) + rest)), &s, &c);
    turn_cos[t][pair] = c * r.factor;
    turn_sin[t][pair] = s * r.factor;
  }
  __syncthreads();
  const int units = (r.q_heads + 2 * a.num_kv_heads) * kParts, per_block = (units + int(gridDim.y) - 1) / int(gridDim.y);
  const int first = int(blockIdx.y) * per_block, mine = first + per_block < units ? per_block : units - first;
  // items: the units of the first token, of the second ...; a thread has every 256th of them
  for (int t = 0, unit = tid;; unit += 256) {
    while (unit >= mine && t < TOKENS) unit -= mine, ++t;   // (mine > 0)
    if (t >= TOKENS) break;
    const Kv16Token x = tokens[t];
    const int at = first + unit, part = at % kParts, row = t0 + t;
    int head = at / kParts;
    const bool is_q = head < r.q_heads;
    if (!x.valid || (!is_q && x.place < 0)) continue;
    const char* src;
    char* dst;
    bool turned = part * 16 < r.rotary;
    if (is_q) {
      src = r.q + row * r.q_stride_t + head * r.q_stride_h;
      dst = r.q_out + (int64_t(row) * r.q_heads + head) * (2 * HD);
    } else {
      head -= r.q_heads;
      const bool is_v = head >= a.num_kv_heads;
      if (is_v) head -= a.num_kv_heads, turned = false;
      src = (is_v ? r.v : r.k) + row * r.stride_t + head * r.stride_h;
      dst = (is_v ? r.v_pool : r.k_pool) + x.place + int64_t(head) * a.page_size * (2 * HD);
    }
    const bool halves = turned && !r.interleaved;
    const int at0 = halves ? part * 16 : part * 32, at1 = halves ? r.rotary + part * 16 : part * 32 + 16;   // bytes
    u32x4 lo = *reinterpret_cast<const u32x4*>(src + at0), hi = *reinterpret_cast<const u32x4*>(src + at1);
    if (turned) {
      const float *cs = &turn_cos[t][part * 8], *sn = &turn_sin[t][part * 8];
      if (halves) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const float x0 = low_of<BF16>(lo[w]), x1 = high_of<BF16>(lo[w]), y0 = low_of<BF16>(hi[w]), y1 = high_of<BF16>(hi[w]);
          lo[w] = pack_pair<BF16>(x0 * cs[2 * w] - y0 * sn[2 * w], x1 * cs[2 * w + 1] - y1 * sn[2 * w + 1]);
          hi[w] = pack_pair<BF16>(y0 * cs[2 * w] + x0 * sn[2 * w], y1 * cs[2 * w + 1] + x1 * sn[2 * w + 1]);
        }
      } else {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const float x0 = low_of<BF16>(lo[w]), y0 = high_of<BF16>(lo[w]), x1 = low_of<BF16>(hi[w]), y1 = high_of<BF16>(hi[w]);
          lo[w] = pack_pair<BF16>(x0 * cs[w] - y0 * sn[w], y0 * cs[w] + x0 * sn[w]);
          hi[w] = pack_pair<BF16>(x1 * cs[w + 4] - y1 * sn[w + 4], y1 * cs[w + 4] + x1 * sn[w + 4]);
        }
      }
    }
    *reinterpret_cast<u32x4*>(dst + at0) = lo;
    *reinterpret_cast<u32x4*>(dst + at1) = hi;
  }
}

int check_kv16_cache(const cocktail_kv16_cache* c) {
  if (!c) return fail(COCKTAIL_EINVAL, "cache is NULL");
  if (int rc = check_page_table(&c->pages)) return rc;
  if (c->num_kv_heads < 1 || c->num_kv_heads > 1024) return fail(COCKTAIL_EINVAL, "num_kv_heads %d is not in 1 .. 1024", c->num_kv_heads);
  if (c->head_dim != 64 && c->head_dim != 128)
    return fail(COCKTAIL_EUNSUPPORTED, "kernels are built for head_dim 64 and 128, got %d", c->head_dim);
  if (c->dtype != COCKTAIL_FP16 && c->dtype != COCKTAIL_BF16) return fail(COCKTAIL_EINVAL, "dtype %d is neither COCKTAIL_FP16 nor COCKTAIL_BF16", c->dtype);
  if (c->pages.page_size % 16 || c->pages.page_size > kMostPageSize)
    return fail(COCKTAIL_EINVAL, "page_size %d is not a multiple of 16 up to %d", c->pages.page_size, kMostPageSize);
  // (positions and the numbers of keys a little behind the last one are ints)
  if (int64_t(c->pages.table_stride) * c->pages.page_size > (int64_t(1) << 31) - 256)
    return fail(COCKTAIL_EINVAL, "table_stride * page_size must be at most 2^31 - 256 for the cache");
  if (!c->k || !c->v) return fail(COCKTAIL_EINVAL, "the pools must not be NULL");
  if ((reinterpret_cast<uintptr_t>(c->k) | reinterpret_cast<uintptr_t>(c->v)) & 15) return fail(COCKTAIL_EALIGN, "the pools must be 16-byte aligned");
  return COCKTAIL_OK;
}

int check_kv16_rows(const cocktail_kv16_cache* c, const void* x, const void* y, int64_t stride_t, int64_t stride_h, int64_t total, int heads) {
  if (total && (!x || !y)) return fail(COCKTAIL_EINVAL, "the rows must not be NULL");
  if ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(y)) & 15) return fail(COCKTAIL_EALIGN, "the rows must be 16-byte aligned");
  if (stride_t < 0 || stride_h < 0 || stride_t % 8 || stride_h % 8 || stride_t > (int64_t(1) << 31) || stride_h > (int64_t(1) << 31))
    return fail(COCKTAIL_EINVAL, "strides must be multiples of 8 in 0 .. 2^31");
  if (heads > 1 && stride_h < c->head_dim) return fail(COCKTAIL_EINVAL, "heads overlap: stride_h %lld", (long long)stride_h);
  if (total > 1 && stride_t < c->head_dim) return fail(COCKTAIL_EINVAL, "rows overlap: stride_t %lld", (long long)stride_t);
  return COCKTAIL_OK;
}

int check_kv16_batch(const cocktail_kv16_cache* c, int64_t total, const int32_t* starts, PagedBatch* a) {
  if (total < 0 || total > (int64_t(1) << 30)) return fail(COCKTAIL_EINVAL, "total %lld is not in 0 .. 2^30", (long long)total);
  if (reinterpret_cast<uintptr_t>(starts) & 3) return fail(COCKTAIL_EALIGN, "starts must be 4-byte aligned");
  if (!starts && total % c->pages.num_seqs)
    return fail(COCKTAIL_EINVAL, "without starts the rows (%lld) must be a multiple of the sequences (%d)", (long long)total, c->pages.num_seqs);
  const cocktail_page_table& p = c->pages;
  *a = {static_cast<char*>(c->k), p.table, p.seq_lens, starts, p.num_seqs, p.table_stride, p.page_size, p.num_pages, c->num_kv_heads,
        int32_t(total), int32_t(total), int32_t(total / p.num_seqs)};
  return COCKTAIL_OK;
}

}  // namespace cocktail

using namespace cocktail;

extern "C" int cocktail_kv16_append(const cocktail_kv16_cache* cache, const void* k, const void* v, int64_t stride_t, int64_t stride_h,
                                    int64_t total, const int32_t* starts, const cocktail_rotation* rotation, const int32_t* positions,
                                    const void* q, int32_t num_q_heads, int64_t q_stride_t, int64_t q_stride_h, void* q_out, void* stream) {
  PagedBatch a;
  if (int rc = check_kv16_cache(cache)) return rc;
  if (int rc = check_kv16_rows(cache, k, v, stride_t, stride_h, total, cache->num_kv_heads)) return rc;
  if (int rc = check_kv16_batch(cache, total, starts, &a)) return rc;
  const int hd = cache->head_dim;
  if (rotation) {
    if (!rotation->inv_freq) return fail(COCKTAIL_EINVAL, "inv_freq is NULL");
    if (reinterpret_cast<uintptr_t>(rotation->inv_freq) & 7) return fail(COCKTAIL_EALIGN, "inv_freq must be 8-byte aligned");
    if (rotation->rotary_dim < 16 || rotation->rotary_dim > hd || rotation->rotary_dim % 16)
      return fail(COCKTAIL_EUNSUPPORTED, "rotary_dim %d is not a multiple of 16 up to %d", rotation->rotary_dim, hd);
    if (rotation->interleaved != 0 && rotation->interleaved != 1) return fail(COCKTAIL_EINVAL, "interleaved must be 0 or 1");
    if (!std::isfinite(rotation->factor)) return fail(COCKTAIL_EINVAL, "factor must be finite");
  }
  if (reinterpret_cast<uintptr_t>(positions) & 3) return fail(COCKTAIL_EALIGN, "positions must be 4-byte aligned");
  if (positions && !rotation) return fail(COCKTAIL_EINVAL, "positions are those of a rotation");
  if (q) {
    if (!rotation) return fail(COCKTAIL_EINVAL, "q is for a rotation");
    if (num_q_heads < 1 || num_q_heads > 65536) return fail(COCKTAIL_EINVAL, "num_q_heads %d is not in 1 .. 65536", num_q_heads);
    if (!q_out) return fail(COCKTAIL_EINVAL, "q_out is NULL");
    if (int rc = check_kv16_rows(cache, q, q_out, q_stride_t, q_stride_h, total, num_q_heads)) return rc;
    if (q == q_out && ((num_q_heads > 1 && q_stride_h != hd) || (total > 1 && q_stride_t != int64_t(num_q_heads) * hd)))
      return fail(COCKTAIL_EINVAL, "q can be rotated in place only where it is contiguous");
  } else if (num_q_heads != 0 || q_out) {
    return fail(COCKTAIL_EINVAL, "without q there are no query heads and no q_out");
  }
  if (!total) return COCKTAIL_OK;
  const int64_t pool_bytes = kv16_pool_bytes(cache);
  if (overlap(cache->k, pool_bytes, cache->v, pool_bytes)) return fail(COCKTAIL_EINVAL, "the pools overlap");
  if (q) {
    const cocktail_page_table& pt = cache->pages;
    const int64_t rows = kv16_extent(cache, stride_t, stride_h, total, cache->num_kv_heads);
    const MemoryRange written[] = {{q_out, 2 * total * num_q_heads * hd}};
    const MemoryRange others[] = {{q, q == q_out ? 0 : kv16_extent(cache, q_stride_t, q_stride_h, total, num_q_heads)}, {k, rows}, {v, rows}, {cache->k, pool_bytes}, {cache->v, pool_bytes},
                                  {pt.table, 4 * int64_t(pt.num_seqs) * pt.table_stride}, {pt.seq_lens, 4 * int64_t(pt.num_seqs)}, {pt.status, 16},
                                  {starts, starts ? 4 * (int64_t(pt.num_seqs) + 1) : 0}, {positions, positions ? 4 * total : 0},
                                  {rotation->inv_freq, 4 * int64_t(rotation->rotary_dim)}};
    if (overlap(written, others)) return fail(COCKTAIL_EINVAL, "q_out overlaps with what the call reads or stores to");
  }
  Kv16Rows r = {};
  r.k = static_cast<const char*>(k);
  r.v = static_cast<const char*>(v);
  r.q = static_cast<const char*>(q);
  r.k_pool = static_cast<char*>(cache->k);
  r.v_pool = static_cast<char*>(cache->v);
  r.q_out = static_cast<char*>(q_out);
  r.stride_t = 2 * stride_t;
  r.stride_h = 2 * stride_h;
  r.q_stride_t = 2 * q_stride_t;
  r.q_stride_h = 2 * q_stride_h;
  r.positions = positions;
  r.status = cache->pages.status;
  if (rotation) {
    r.inv_freq = rotation->inv_freq;
    r.rotary = rotation->rotary_dim;
    r.interleaved = rotation->interleaved;
    r.factor = rotation->factor;
  }
  r.q_heads = num_q_heads;
  // Four tokens share what is to be found out for them where that leaves workgroups enough, else workgroups share a token.  (32K tokens of 48 heads: 2, 4, 8,
  // 16 tokens 161, 154, 165, 180 us, and with two or four items of a thread on their way instead of one 164 and 173: it is the order in which the memory is
  // touched; without the caches 157 .. 170, and neighbouring pairs, which write half lines, 287 instead of 184.)
  const int tokens = total >= 2048 ? 4 : 1;
  const int parts = tokens == 1 ? ((num_q_heads + 2 * cache->num_kv_heads) * (hd / 16) + 255) / 256 : 1;
  const int64_t blocks = (total + tokens - 1) / tokens;
  if (blocks * parts >= (int64_t(1) << 24)) return fail(COCKTAIL_EINVAL, "append of %lld rows is more than one launch takes", (long long)total);
  typedef void (*Kernel)(PagedBatch, Kv16Rows);
  static const Kernel kernels[2][2][2] = {{{kv16_append_kernel<64, false, 1>, kv16_append_kernel<64, false, 4>}, {kv16_append_kernel<64, true, 1>, kv16_append_kernel<64, true, 4>}},
                                          {{kv16_append_kernel<128, false, 1>, kv16_append_kernel<128, false, 4>}, {kv16_append_kernel<128, true, 1>, kv16_append_kernel<128, true, 4>}}};
  const size_t lds = starts ? (a.num_seqs + 1) * sizeof(int32_t) : 0;
  const hipError_t e = launch_lds(kernels[hd == 128][cache->dtype == COCKTAIL_BF16][tokens > 1], dim3(uint32_t(blocks), uint32_t(parts)), dim3(256), lds, static_cast<hipStream_t>(stream), a, r);
  if (e != hipSuccess) return fail(COCKTAIL_EHIP, "append launch failed: %s", hipGetErrorString(e));
  return COCKTAIL_OK;
}
