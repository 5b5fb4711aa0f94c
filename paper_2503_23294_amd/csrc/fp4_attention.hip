// cocktail_fp4_attention: which kernel serves which sequences, the C entry.
#include <hip/hip_runtime.h>

#include <cmath>
#include <type_traits>

#include "fp4_decode_impl.h"
#include "fp4_tiles_impl.h"

using namespace cocktail;

namespace {

// What a call launches, from what the host knows: bounds, no lengths.
struct Split {
  bool decode, whole, tiles;
  int rows, row_tiles, workers, tile_waves, tile_blocks, splits;
  int64_t active;   // sequences that have queries at most
  size_t prefix_bytes, part_rows, tile_rows, bytes;
};

Split split_of(const cocktail_fp4_cache* c, int rep, int64_t total, int64_t max_new, int64_t max_len, bool uniform) {
  Split s = {};
  const int64_t capacity = int64_t(c->pages.table_stride) * c->pages.page_size;
  if (max_len <= 0 || max_len > capacity) max_len = capacity;
  const int64_t most_rows = max_new * rep;
  s.active = c->pages.num_seqs < total ? c->pages.num_seqs : total;
  // A batch may hold sequences for either kernel, unless all have the same number of queries or the others cannot have so many that one is left with
  // few: then the tile kernel has them all, whatever their numbers are, and two launches with nothing to do are saved (5 us each by themselves, 1 to 9 us of a call of 0.8 ms).
  s.tiles = most_rows > kDecodeRows;
  const int64_t least = total - (int64_t(c->pages.num_seqs) - 1) * max_new;
  s.decode = !s.tiles || (!uniform && rep <= kDecodeRows && least * rep <= kDecodeRows);
  s.rows = int(most_rows < kDecodeRows ? most_rows : kDecodeRows);
  s.row_tiles = (s.rows + 15) / 16;
  if (s.decode) {
    // Two waves per SIMD of 256 compute units (128K, 40 heads: 1024 waves 116 us, 2048 111, half as many again 113; 8 x 16K, 32 rows: 1024 waves 47.5 us, 2048
    // 44.4), one where a wave has three or four operands of queries and needs all registers; and four units at
    // least for a wave, at half a microsecond each: with fewer the states cost more than that (8 heads, 16K: 2, 4, 8 units 20.8, 15.4, 15.0 us;
    // 2K: 10.2, 10.9, 14.7).
    const int64_t seqs = s.active;
    const int64_t units = seqs * ((max_len + kUnit - 1) / kUnit) * c->num_kv_heads;
    int64_t workers = (units + 3) / 4;
    const int64_t fill = s.row_tiles <= 2 ? 2048 : 1024;
    workers = workers > fill ? fill : workers < 4 ? 4 : (workers + 3) / 4 * 4;
    s.workers = int(workers);
    // A workgroup per segment and no merge where contexts are short: up to 2K (8 heads: 1000, 2048 tokens 12.2, 11.5 us in two launches,
    // 6.7, 9.4 in one; 4096: 11.9 and 15.3), and up to 6K where the segments fill the chip by themselves (128, 256, 512, 1024 of 4096 tokens:
    // 23.0, 32.6, 57.3, 104.7 and 19.6, 25.5, 46.7, 101.5; of 8192 the same within 3 %, but there one long sequence among short ones would be waited for).
    const int64_t segments = seqs * c->num_kv_heads;
    s.whole = s.row_tiles == 1 && max_len <= (segments >= 128 ? 6144 : 2048);
    if (s.whole) workers = 0;
    s.prefix_bytes = (size_t(c->pages.num_seqs) + 1 + 63) / 64 * 256;
    s.part_rows = 2 * size_t(workers) * s.rows;
  }
  s.splits = 1;
  if (s.tiles) {
    const int64_t seqs = c->pages.num_seqs;
    // Eight waves share what it takes to bring the keys into LDS where that leaves a workgroup for every compute unit and the rows see about as
    // many keys each (2048 tokens of 4 x 8 heads behind 30K: four waves 1180 us, eight 1135); else four, whose smaller pieces
    // leave less to wait for at the end (whole prompts of 8190 and 4095 tokens, 32 heads: 778 us, and 797 with eight).
    s.tile_waves = total * rep * c->num_kv_heads >= 256 * 256 && most_rows > 128 && max_len >= 2 * max_new ? 8 : 4;
    const int64_t tile_rows = 32 * s.tile_waves;
    s.tile_blocks = int(uniform ? seqs * ((most_rows + tile_rows - 1) / tile_rows) : total * rep / tile_rows + (seqs < total ? seqs : total));
    const int64_t have = int64_t(s.tile_blocks) * c->num_kv_heads;
    // Parts only where there are fewer workgroups than run at a time (one on a compute unit with eight waves, two with four): as many as make
    // the last round of them fullest, each of 512 keys at least.
    const int64_t at_once = s.tile_waves == 8 ? 256 : 512;
    const int64_t longest = (max_len + 511) / 512;
    double best = 0;
    for (int64_t parts = 1; parts <= 64 && parts <= longest && (parts == 1 || have * (parts - 1) < at_once); ++parts) {
      const double time = double((have * parts + at_once - 1) / at_once) / double(parts) + 0.01 * double(parts);
      if (parts == 1 || time < best) best = time, s.splits = int(parts);
    }
    if (s.splits > 1) s.tile_rows = size_t(s.splits) * size_t(total) * c->num_kv_heads * rep;
  }
  s.bytes = s.prefix_bytes + (s.part_rows + s.tile_rows) * (c->head_dim + 4) * sizeof(float) + 64;
  return s;
}

int check_attention(const cocktail_fp4_cache* c, int32_t num_q_heads, int64_t total, int32_t max_new) {
  if (int rc = check_fp4_cache(c)) return rc;
  if (num_q_heads < 1 || num_q_heads % c->num_kv_heads)
    return fail(COCKTAIL_EINVAL, "num_q_heads %d is not a positive multiple of num_kv_heads %d", num_q_heads, c->num_kv_heads);
  if (num_q_heads / c->num_kv_heads > COCKTAIL_MAX_Q_PER_KV)
    return fail(COCKTAIL_EUNSUPPORTED, "num_q_heads / num_kv_heads = %d, at most %d", num_q_heads / c->num_kv_heads, COCKTAIL_MAX_Q_PER_KV);
  if (total < 0 || total * num_q_heads > (int64_t(1) << 30)) return fail(COCKTAIL_EINVAL, "total %lld is negative or too many for %d heads", (long long)total, num_q_heads);
  if (total && (max_new < 1 || max_new > total)) return fail(COCKTAIL_EINVAL, "max_new %d is not in 1 .. total (%lld)", max_new, (long long)total);
  const int64_t capacity = int64_t(c->pages.table_stride) * c->pages.page_size;
  if (double(c->pages.num_seqs) * ((capacity + kUnit - 1) / kUnit) * c->num_kv_heads > 8.5e8)   // (costs, up to five times that, are 32 bits wide)
    return fail(COCKTAIL_EINVAL, "%d sequences of up to %lld tokens are too many for one call", c->pages.num_seqs, (long long)capacity);
  return COCKTAIL_OK;
}

}  // namespace

extern "C" int cocktail_fp4_attention_workspace(const cocktail_fp4_cache* cache, int32_t num_q_heads, int64_t total, int32_t max_new,
                                                int32_t max_len, int32_t uniform, size_t* bytes) {
  if (!bytes) return fail(COCKTAIL_EINVAL, "bytes is NULL");
  if (int rc = check_attention(cache, num_q_heads, total, max_new)) return rc;
  *bytes = total ? split_of(cache, num_q_heads / cache->num_kv_heads, total, max_new, max_len, uniform != 0).bytes : 0;
  return COCKTAIL_OK;
}

extern "C" int cocktail_fp4_attention(const cocktail_fp4_cache* cache, int32_t num_q_heads, const void* q, int32_t dtype, int64_t stride_t,
                                      int64_t stride_h, int64_t total, const int32_t* starts, int32_t max_new, int32_t max_len,
                                      float sm_scale, void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  PagedAttention a = {};
  if (int rc = check_attention(cache, num_q_heads, total, max_new)) return rc;
  if (int rc = check_fp4_rows(cache, q, out, dtype, stride_t, stride_h, total, starts, num_q_heads, &a.batch)) return rc;
  if (!total) return COCKTAIL_OK;
  if (!starts && max_new != total / cache->pages.num_seqs)
    return fail(COCKTAIL_EINVAL, "without starts max_new (%d) must be total / num_seqs (%lld)", max_new, (long long)(total / cache->pages.num_seqs));
  if (std::isnan(sm_scale) || std::isinf(sm_scale)) return fail(COCKTAIL_EINVAL, "sm_scale must be finite");
  if (reinterpret_cast<uintptr_t>(lse) & 3) return fail(COCKTAIL_EALIGN, "lse must be 4-byte aligned");
  if (!workspace) return fail(COCKTAIL_EINVAL, "workspace is NULL");
  if (reinterpret_cast<uintptr_t>(workspace) & 15) return fail(COCKTAIL_EALIGN, "workspace must be 16-byte aligned");
  const int hd = cache->head_dim;
  a.rep = num_q_heads / cache->num_kv_heads;
  const Split s = split_of(cache, a.rep, total, max_new, max_len, !starts);
  if (workspace_bytes < s.bytes) return fail(COCKTAIL_ENOSPACE, "workspace has %zu bytes, %zu are needed", workspace_bytes, s.bytes);
  a.batch.max_new = max_new;
  a.q = static_cast<const char*>(q);
  a.out = static_cast<char*>(out);
  a.lse = lse;
  a.stride_t = 2 * stride_t;
  a.stride_h = 2 * stride_h;
  a.bf16 = dtype == COCKTAIL_BF16;
  a.scale = (sm_scale > 0.f ? sm_scale : 1.f / std::sqrt(float(hd))) * kLog2e;
  a.rows = s.rows;
  a.workers = s.workers;
  a.decode_rows = s.decode ? kDecodeRows : 0;
  a.splits = s.splits;
  char* w = static_cast<char*>(workspace);
  a.prefix = reinterpret_cast<int32_t*>(w);
  w += s.prefix_bytes;
  a.part_o = reinterpret_cast<float*>(w);
  w += s.part_rows * hd * sizeof(float);
  a.tile_o = reinterpret_cast<float*>(w);
  w += s.tile_rows * hd * sizeof(float);
  a.part_ml = reinterpret_cast<float*>(w);
  w += s.part_rows * 3 * sizeof(float);
  a.tile_ml = reinterpret_cast<float*>(w);

  hipStream_t st = static_cast<hipStream_t>(stream);
  hipError_t e = hipSuccess;
  if (s.decode) {
    typedef void (*Kernel)(PagedAttention);
    static const Kernel kernels[2][4] = {{fp4_decode_kernel<64, 1, false>, fp4_decode_kernel<64, 2, false>, fp4_decode_kernel<64, 3, false>, fp4_decode_kernel<64, 4, false>},
                                         {fp4_decode_kernel<128, 1, false>, fp4_decode_kernel<128, 2, false>, fp4_decode_kernel<128, 3, false>, fp4_decode_kernel<128, 4, false>}};
    const int64_t segments = s.active * cache->num_kv_heads;
    // Few segments leave most of the chip idle while their compute units convert and multiply: four workgroups to a segment, each for a quarter of the
    // channels of V, all with the logits of their own (8 segments of 1000, 2048 tokens: 7.6, 10.9 -> 6.7, 9.4 us; 32: 7.7, 11.2 -> 6.9, 10.3; 64: 7.9, 11.4 ->
    // 8.0, 14.8, for everything is read four times; halves of 64 channels: the same as whole ones)
    const bool quarters = segments <= 32 && hd == 128;
    if (s.whole)
      e = launch(quarters ? fp4_decode_kernel<128, 1, true, 4> : hd == 128 ? fp4_decode_kernel<128, 1, true> : fp4_decode_kernel<64, 1, true>,
                 dim3(uint32_t(segments) * (quarters ? 4 : 1)), dim3(64 * kWholeWaves), st, a);
    else
      e = launch_lds(kernels[hd == 128][s.row_tiles - 1], dim3(s.workers / kDecodeWaves), dim3(64 * kDecodeWaves), (a.batch.num_seqs + 1) * sizeof(int32_t), st, a);
  }
  if (e == hipSuccess && s.tiles)
    e = launch(s.tile_waves == 8 ? (hd == 128 ? fp4_tile_kernel<128, 8> : fp4_tile_kernel<64, 8>) : (hd == 128 ? fp4_tile_kernel<128, 4> : fp4_tile_kernel<64, 4>),
               dim3(uint32_t(s.tile_blocks) * s.splits * cache->num_kv_heads), dim3(64 * s.tile_waves), st, a);
  if (e == hipSuccess && s.decode && !s.whole) {
    int most_new = kDecodeRows / a.rep < max_new ? kDecodeRows / a.rep : max_new;
    if (int64_t(cache->pages.num_seqs) * most_new > 4 * total) most_new = 0;
    const uint32_t most = uint32_t(most_new ? int64_t(cache->pages.num_seqs) * most_new : total) * num_q_heads;
    // states that a row has, about: many of them are read by many waves at a time (40 rows of 51 states: 8.8 us by four waves, 5.6 by sixteen; 1024 rows of
    // 32: calls of 43.6 us by one wave a row, 36.9 by four; three times as many rows of 16: 60.5 and 62), a few by one
    const int parts = int(s.workers / (s.active * cache->num_kv_heads));
    if (parts >= 16 && most <= 512)
      e = launch(hd == 128 ? merge_decode_kernel<Fp4Cost, 128, 16> : merge_decode_kernel<Fp4Cost, 64, 16>, dim3(most), dim3(1024), st, a, most_new);
    else if (parts >= 12 && most <= 2048)
      e = launch(hd == 128 ? merge_decode_kernel<Fp4Cost, 128, 4> : merge_decode_kernel<Fp4Cost, 64, 4>, dim3(most), dim3(256), st, a, most_new);
    else
      e = launch(hd == 128 ? merge_decode_kernel<Fp4Cost, 128, 1> : merge_decode_kernel<Fp4Cost, 64, 1>, dim3((most + 3) / 4), dim3(256), st, a, most_new);
  }
  if (e == hipSuccess && s.splits > 1)
    e = launch(hd == 128 ? merge_tiles_kernel<Fp4Cost, 128> : merge_tiles_kernel<Fp4Cost, 64>, dim3(uint32_t((total * num_q_heads + 3) / 4)), dim3(256), st, a);
  if (e != hipSuccess) return fail(COCKTAIL_EHIP, "attention launch failed: %s", hipGetErrorString(e));
  return COCKTAIL_OK;
}
