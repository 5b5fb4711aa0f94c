// cocktail_kv16_attention: which kernel serves which sequences, the C entry.
#include <hip/hip_runtime.h>

#include <cmath>
#include <type_traits>

#include "kv16_decode_impl.h"
#include "kv16_tiles_impl.h"

using namespace cocktail;

namespace {

int check_attention(const cocktail_kv16_cache* c, int32_t num_q_heads, int64_t total, int32_t max_new) {
  if (int rc = check_kv16_cache(c)) return rc;
  if (num_q_heads < 1 || num_q_heads % c->num_kv_heads)
    return fail(COCKTAIL_EINVAL, "num_q_heads %d is not a positive multiple of num_kv_heads %d", num_q_heads, c->num_kv_heads);
  if (num_q_heads / c->num_kv_heads > COCKTAIL_MAX_Q_PER_KV)
    return fail(COCKTAIL_EUNSUPPORTED, "num_q_heads / num_kv_heads = %d, at most %d", num_q_heads / c->num_kv_heads, COCKTAIL_MAX_Q_PER_KV);
  if (total < 0 || total > (int64_t(1) << 30) / num_q_heads) return fail(COCKTAIL_EINVAL, "total %lld is negative or too many for %d heads", (long long)total, num_q_heads);
  if (total && (max_new < 1 || max_new > total)) return fail(COCKTAIL_EINVAL, "max_new %d is not in 1 .. total (%lld)", max_new, (long long)total);
  const int64_t capacity = int64_t(c->pages.table_stride) * c->pages.page_size;
  if (double(c->pages.num_seqs) * ((capacity + kUnit - 1) / kUnit) * c->num_kv_heads > 8.5e8)   // (units are numbered in 32 bits)
    return fail(COCKTAIL_EINVAL, "%d sequences of up to %lld tokens are too many for one call", c->pages.num_seqs, (long long)capacity);
  return COCKTAIL_OK;
}

// What a call launches, from what the host knows: bounds, no lengths.
struct Split {
  bool decode, tiles, joins;
  DecodeWork work;
  int rows, row_tiles, workers, tile_waves, tile_blocks, splits;
  int64_t active;   // sequences that have queries at most
  size_t prefix_bytes, part_rows, tile_rows, bytes;
};

Split split_of(const cocktail_kv16_cache* c, int rep, int64_t total, int64_t max_new, int64_t max_len, bool uniform) {
  Split s = {};
  const int64_t capacity = int64_t(c->pages.table_stride) * c->pages.page_size;
  if (max_len <= 0 || max_len > capacity) max_len = capacity;
  const int64_t most_rows = max_new * rep;
  s.active = c->pages.num_seqs < total ? c->pages.num_seqs : total;
  // A batch may hold sequences for either kernel, unless all have the same number of queries or the others cannot have so many that one is left with
  // few: then the tile kernel has them all, whatever their numbers are.
  s.tiles = most_rows > kDecodeRows;
  const int64_t least = total - (int64_t(c->pages.num_seqs) - 1) * max_new;
  s.decode = !s.tiles || (!uniform && rep <= kDecodeRows && least * rep <= kDecodeRows);
  s.rows = int(most_rows < kDecodeRows ? most_rows : kDecodeRows);
  s.row_tiles = (s.rows + 15) / 16;
  if (s.decode) {
    const int64_t units = s.active * ((max_len + kUnit - 1) / kUnit) * c->num_kv_heads;
    // A wave per SIMD of 256 compute units: one has 16 KB on their way at any time, which is enough (128K, 40 heads: 390 us; 64 of up to 4K, 8 kv heads:
    // 512, 768, 1024, 1280, 2048 waves 152, 113, 102, 137, 111).  Of short contexts a wave has one unit, or two where there are more than 512 (2K,
    // 8 heads: 1, 2, 4 units a wave 11.5, 12.5, 14.6; 8K: 18.8, 14.8, 15.7).
    int64_t workers = units <= 512 ? units : units <= 1024 ? 512 : units / 2;
    const int64_t fill = 1024;
    workers = workers > fill ? fill : workers < 4 ? 4 : (workers + 3) / 4 * 4;
    s.workers = int(workers);
    // A workgroup per segment and no merge where contexts are short, of 128 KB of K at most: a compute unit reads no faster (8 heads of 128, 200
    // tokens: two launches 10.0 us, one 7.7; 1000: 11.5, 14.3; 32 sequences of 512: 19.7, 15.2, of 2048: 48.8, 46.5; 24 x 32 heads, 1024: 68.9, 77.8, of 64
    // channels 37.2, 33.0).  Of more rows two launches cost more: 32 rows of 8 heads of 128, 200 and 512 tokens 12.2, 10.1 and 12.7, 12.6, 64 rows of 256 (32
    // sequences, 8 heads) 36.3, 13 and 35, 17; where there are segments for half the compute units, also of longer contexts: 32 rows of 160, 1000 tokens 28.3,
    // 20.1; 64 of 160, 1000, 2000 38, 23; 51, 34.
    const int64_t segments = s.active * c->num_kv_heads;
    const bool whole = max_len * c->head_dim <= 65536 * (segments < 128 || s.row_tiles == 1 ? 1 : s.row_tiles == 2 ? 2 : 3);
    // Shares of workgroups from some 32 units of a workgroup on (64 rows, 512 segments of 2000, 4000 tokens 145, 109; 236, 185; 256 of 1000 44, 36; 8 of 20K: 30,
    // 36; 40 rows, 64 of 300 .. 4000: 27.6, 32).
    s.work = whole ? kWholeSegments : s.row_tiles > 1 && units >= 32 * kComputeUnits ? kGroupShares : kWaveShares;
    if (s.work == kGroupShares) s.workers = int(workers /= kDecodeWaves);
    if (whole) workers = 0;
    // Whether a workgroup's waves leave one state where all have parts of one segment: less to write and to read for the merge, which else takes (2 heads
    // of one kv head, 84K tokens, 880 states) 20.3 us, joined 9.8; 7 of one, 4.7K 7.4, 5.9; 32 of 8, 20K 6.2, 5.2; but 8 of 8, 2K, 64 states 4.8, 4.8.  Of
    // many rows states are large (verification behind 16K, 16 states of 48 rows: both kernels 74.8, 73.5).
    s.joins = s.work == kWaveShares && workers > (s.row_tiles > 1 ? 8 : 64) * segments;
    s.prefix_bytes = (size_t(c->pages.num_seqs) + 1 + 63) / 64 * 256;
    s.part_rows = 2 * size_t(workers) * s.rows;
  }
  s.splits = 1;
  if (s.tiles) {
    const int64_t seqs = c->pages.num_seqs;
    // Eight waves share what it takes to bring the keys into LDS where that leaves a workgroup for every compute unit and the rows see about as
    // many keys each, or else two of them (head_dim 128, us with four and eight: 2048 new of 8192, 8 x 4 heads 253, 245; prompts of 2048, 3000, 4096, 8192
    // tokens with 32, 40, 32, 32 heads 63, 68; 115, 125; 160, 158; 573, 550; head_dim 64 the same within 5 %); else four, whose smaller pieces leave less
    // to wait for at the end.
    s.tile_waves = total * rep * c->num_kv_heads >= 256 * 256 * (max_len >= 2 * max_new ? 1 : 2) && most_rows > 128 ? 8 : 4;
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

}  // namespace

extern "C" int cocktail_kv16_attention_workspace(const cocktail_kv16_cache* cache, int32_t num_q_heads, int64_t total, int32_t max_new,
                                                 int32_t max_len, int32_t uniform, size_t* bytes) {
  if (!bytes) return fail(COCKTAIL_EINVAL, "bytes is NULL");
  if (int rc = check_attention(cache, num_q_heads, total, max_new)) return rc;
  *bytes = total ? split_of(cache, num_q_heads / cache->num_kv_heads, total, max_new, max_len, uniform != 0).bytes : 0;
  return COCKTAIL_OK;
}

extern "C" int cocktail_kv16_attention(const cocktail_kv16_cache* cache, int32_t num_q_heads, const void* q, int64_t stride_t, int64_t stride_h,
                                       int64_t total, const int32_t* starts, int32_t max_new, int32_t max_len, float sm_scale, void* out,
                                       float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  Kv16Attention args = {};
  PagedAttention& a = args.p;
  if (int rc = check_attention(cache, num_q_heads, total, max_new)) return rc;
  if (int rc = check_kv16_rows(cache, q, out, stride_t, stride_h, total, num_q_heads)) return rc;
  if (int rc = check_kv16_batch(cache, total, starts, &a.batch)) return rc;
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
  const int64_t rows = total * num_q_heads;
  const bool in_place = q == out && (num_q_heads == 1 || stride_h == hd) && (total == 1 || stride_t == int64_t(num_q_heads) * hd);
  const cocktail_page_table& pt = cache->pages;
  const int64_t q_bytes = kv16_extent(cache, stride_t, stride_h, total, num_q_heads), pool_bytes = kv16_pool_bytes(cache);
  const MemoryRange written[] = {{out, 2 * rows * hd}, {lse, lse ? 4 * rows : 0}, {workspace, int64_t(s.bytes)}};
  const MemoryRange read[] = {{q, in_place ? 0 : q_bytes}, {cache->k, pool_bytes}, {cache->v, pool_bytes}, {pt.table, 4 * int64_t(pt.num_seqs) * pt.table_stride},
                              {pt.seq_lens, 4 * int64_t(pt.num_seqs)}, {starts, starts ? 4 * (int64_t(pt.num_seqs) + 1) : 0}};
  if (overlap(written, read)) return fail(COCKTAIL_EINVAL, "out, lse and workspace overlap with each other or with what the call reads");
  // A wave of the merge per row, fewer than 2^32 threads; refused also where the call needs no merge, so that the limit does not hang on max_len.  (What
  // check_attention and the numbers of sequences and heads leave keeps the other launches below that.)
  if (s.decode && int64_t(cache->pages.num_seqs) * s.rows * cache->num_kv_heads >= int64_t(1) << 26)
    return fail(COCKTAIL_EINVAL, "%d sequences of %d heads with up to %d rows each are too many for one call", cache->pages.num_seqs, cache->num_kv_heads, s.rows);
  a.batch.max_new = max_new;
  args.v_pool = static_cast<const char*>(cache->v);
  a.q = static_cast<const char*>(q);
  a.out = static_cast<char*>(out);
  a.lse = lse;
  a.stride_t = 2 * stride_t;
  a.stride_h = 2 * stride_h;
  a.bf16 = cache->dtype == COCKTAIL_BF16;
  a.scale = (sm_scale > 0.f ? sm_scale : 1.f / std::sqrt(float(hd))) * kLog2e;
  a.rows = s.rows;
  a.workers = s.workers;
  a.splits = s.splits;
  a.joins = s.joins;
  a.decode_rows = s.decode ? kDecodeRows : 0;
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

  typedef void (*Kernel)(Kv16Attention);
  hipStream_t st = static_cast<hipStream_t>(stream);
  hipError_t e = hipSuccess;
  if (s.decode) {
    // by head_dim, type and operands of rows
#define COCKTAIL_ROWS(hd, bf16, work, one) {one, kv16_decode_kernel<hd, bf16, 2, work>, kv16_decode_kernel<hd, bf16, 3, work>, kv16_decode_kernel<hd, bf16, 4, work>}
#define COCKTAIL_ONE(hd, bf16, work) COCKTAIL_ROWS(hd, bf16, work, (kv16_decode_kernel<hd, bf16, 1, work>))
    static const Kernel kernels[3][2][2][4] = {
        {{COCKTAIL_ONE(64, false, kWaveShares), COCKTAIL_ONE(64, true, kWaveShares)}, {COCKTAIL_ONE(128, false, kWaveShares), COCKTAIL_ONE(128, true, kWaveShares)}},
        {{COCKTAIL_ROWS(64, false, kGroupShares, nullptr), COCKTAIL_ROWS(64, true, kGroupShares, nullptr)},
         {COCKTAIL_ROWS(128, false, kGroupShares, nullptr), COCKTAIL_ROWS(128, true, kGroupShares, nullptr)}},
        {{COCKTAIL_ONE(64, false, kWholeSegments), COCKTAIL_ONE(64, true, kWholeSegments)}, {COCKTAIL_ONE(128, false, kWholeSegments), COCKTAIL_ONE(128, true, kWholeSegments)}}};
#undef COCKTAIL_ONE
#undef COCKTAIL_ROWS
    const Kernel kernel = kernels[s.work][hd == 128][a.bf16][s.row_tiles - 1];
    if (s.work == kWholeSegments) e = launch(kernel, dim3(uint32_t(s.active * cache->num_kv_heads)), dim3(64 * whole_waves(s.row_tiles)), st, args);
    else
      e = launch_lds(kernel, dim3(s.work == kGroupShares ? s.workers : s.workers / kDecodeWaves), dim3(64 * kDecodeWaves), (a.batch.num_seqs + 1) * sizeof(int32_t), st,
                     args);
  }
  if (e == hipSuccess && s.tiles) {
    static const Kernel kernels[2][2][2] = {{{kv16_tile_kernel<64, false, 4>, kv16_tile_kernel<64, false, 8>}, {kv16_tile_kernel<64, true, 4>, kv16_tile_kernel<64, true, 8>}},
                                            {{kv16_tile_kernel<128, false, 4>, kv16_tile_kernel<128, false, 8>}, {kv16_tile_kernel<128, true, 4>, kv16_tile_kernel<128, true, 8>}}};
    e = launch(kernels[hd == 128][a.bf16][s.tile_waves == 8], dim3(uint32_t(s.tile_blocks) * s.splits * cache->num_kv_heads), dim3(64 * s.tile_waves), st, args);
  }
  if (e == hipSuccess && s.decode && s.work != kWholeSegments) {
    int most_new = kDecodeRows / a.rep < max_new ? kDecodeRows / a.rep : max_new;
    if (int64_t(cache->pages.num_seqs) * most_new > 4 * total) most_new = 0;
    const uint32_t most = uint32_t(most_new ? int64_t(cache->pages.num_seqs) * most_new : total) * num_q_heads;
    // States that a row has, about: one for a share, or, where workgroups leave one, for their waves' shares together.  Many of them are read by many waves at a
    // time, a few by one (calls on contexts of 16384 tokens, heads of 128, us with 1, 4, 16 waves: 128 states of 1, 16, 64 rows 24.5, 13.2, 12.5; 26.4, 15.0, 13.9;
    // 32.7, 21.1, 20.5; 64 of 4, 64, 256 rows 18.5, 13.2, 13.2; 19.9, 14.2, 14.4; 33.4, 29.9, 29.9; 32 of 8, 512 rows 21.8, 18.9, 19.8; 50.4, 49.3, 51.5; 16 of 256, 1024
    // rows 86.2, 85.5, 86.4; 90.8, 91.1, 97.4; 12 of 340, 1360 rows 112.5, 112.1, 114.5; 118.4, 119.9, 128.1; 8 of 1024 rows 49.5, 50.3, 55.1).
    const int states = int(s.workers / (s.active * cache->num_kv_heads) / (a.joins ? kDecodeWaves : 1));
    if (states >= 96 && most <= 512)
      e = launch(hd == 128 ? merge_decode_kernel<Kv16Cost, 128, 16> : merge_decode_kernel<Kv16Cost, 64, 16>, dim3(most), dim3(1024), st, a, most_new);
    else if (states >= 10 && most <= 1024)
      e = launch(hd == 128 ? merge_decode_kernel<Kv16Cost, 128, 4> : merge_decode_kernel<Kv16Cost, 64, 4>, dim3(most), dim3(256), st, a, most_new);
    else
      e = launch(hd == 128 ? merge_decode_kernel<Kv16Cost, 128, 1> : merge_decode_kernel<Kv16Cost, 64, 1>, dim3((most + 3) / 4), dim3(256), st, a, most_new);
  }
  if (e == hipSuccess && s.splits > 1)
    e = launch(hd == 128 ? merge_tiles_kernel<Kv16Cost, 128> : merge_tiles_kernel<Kv16Cost, 64>, dim3(uint32_t((total * num_q_heads + 3) / 4)), dim3(256), st, a);
  if (e != hipSuccess) return fail(COCKTAIL_EHIP, "attention launch failed: %s", hipGetErrorString(e));
  return COCKTAIL_OK;
}
