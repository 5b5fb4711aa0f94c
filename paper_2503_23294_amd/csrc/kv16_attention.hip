// cocktail_kv16_attention: which kernel serves which sequences, the C entry.
#include <hip/hip_runtime.h>

#include <cmath>
#include <type_traits>

#include "kv16_decode_impl.h"

namespace cocktail {

// A wave has sixteen query rows (new tokens x query heads of a kv head) of one (sequence, kv head) and walks over all of their keys, 32 at a time.
// S^T = K Q^T leaves a lane with one query row and the tokens 4 j + x of two tiles of sixteen, which is the operand of O^T = V^T P^T with tokens numbered accordingly.
template <int HD, bool BF16>
__global__ __launch_bounds__(64) void kv16_rows_kernel(Kv16Attention args) {
  constexpr int kSteps = HD / 32, kChannelTiles = HD / 16;
  const PagedAttention& a = args.p;
  const PagedBatch& bt = a.batch;
  const int lane = threadIdx.x, c16 = lane & 15, j = lane >> 4;
  const int h = blockIdx.x % bt.num_kv_heads, number = blockIdx.x / bt.num_kv_heads;
  // which rows
  int b = -1, tile = 0, run = 0;
  for (int base = 0; base < bt.num_seqs && b < 0; base += 64) {
    const int count = base + lane < bt.num_seqs ? paged_span(bt, base + lane).count * a.rep : 0;
    const int n = count > a.decode_rows ? (count + 15) >> 4 : 0;
    const int upto = wave_prefix(n);
    const uint64_t mask = __ballot(number >= run + upto - n && number < run + upto);
    if (mask) {
      const int at = __builtin_ctzll(mask);
      b = base + at;
      tile = number - run - __builtin_amdgcn_readlane(upto - n, at);
    }
    run += __builtin_amdgcn_readlane(upto, 63);
  }
  if (b < 0) return;
  const PagedSpan span = paged_span(bt, b);
  const int all = paged_len(bt, b), len = paged_held(bt, all);
  const PagedSeq seq = {span.first, span.count, len, all - span.count};
  const int rows = span.count * a.rep, r = tile * 16 + c16, i = r / a.rep;
  const bool live = r < rows;
  const int last_row = (tile * 16 + 16 < rows ? tile * 16 + 16 : rows) - 1;
  const int most = seen_by(seq, last_row / a.rep), lim = live ? seen_by(seq, i) : 0;

  u32x4 q[kSteps] = {};
  if (live) {
    const char* src = a.q + (span.first + i) * a.stride_t + (h * a.rep + r - i * a.rep) * a.stride_h + j * 16;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) q[s] = *reinterpret_cast<const u32x4*>(src + s * 64);
  }
  const float c = fmaxf(a.scale, 1.2e-38f);
  float m = kNoMax, lsum = 0.f;
  f32x4 l = {}, o[kChannelTiles] = {};
  const int P = bt.page_size;
  const int64_t run_bytes = int64_t(P) * (2 * HD);
  for (int tok0 = 0; tok0 < most; tok0 += kUnit) {
    f32x4 s[2] = {};
    u32x4 v[8];
    int ok[2];
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const int t = tok0 + 16 * y, at = t < len ? t : 0;   // (len > 0 here)
      const int page = bt.table[int64_t(b) * bt.table_stride + at / P];
      ok[y] = uint32_t(page) < uint32_t(bt.num_pages) && t < len;
      const int64_t base = (int64_t(ok[y] ? page : 0) * bt.num_kv_heads + h) * run_bytes + int64_t(at % P) * (2 * HD);
      const char* k = bt.pool + base + c16 * (2 * HD) + j * 16;
#pragma unroll
      for (int st = 0; st < kSteps; ++st) s[y] = product16<BF16>(*reinterpret_cast<const u32x4*>(k + st * 64), q[st], s[y]);
      const char* src = args.v_pool + base + c16 * (HD / 8);
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        u32x4& d = v[4 * y + x];
        const char* p = src + (4 * j + x) * (2 * HD);
        if constexpr (HD == 128) {
          d = *reinterpret_cast<const u32x4*>(p);
        } else {
          const u32x2 w = *reinterpret_cast<const u32x2*>(p);
          d = u32x4{w[0], w[1], 0, 0};
        }
        if (!(ok[y] && t + 4 * j + x < len)) d = u32x4{};   // what no token has been stored to may be no number
      }
    }
    float top = kNoMax;
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      const int tok = tok0 + 16 * (x >> 2) + 4 * j + (x & 3);
      s[x >> 2][x & 3] = ok[x >> 2] && tok < lim ? s[x >> 2][x & 3] * c : -__builtin_inff();
      top = fmaxf(top, s[x >> 2][x & 3]);
    }
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    const float raised = fmaxf(m, top), alpha = __builtin_amdgcn_exp2f(m - raised);
    m = raised;
    lsum *= alpha;
    l *= alpha;
#pragma unroll
    for (int ct = 0; ct < kChannelTiles; ++ct) o[ct] *= alpha;
    float w[8];
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      w[x] = __builtin_amdgcn_exp2f(s[x >> 2][x & 3] - m);
      lsum += w[x];
    }
    const u32x4 p = {pack_weights<BF16>(w[0], w[1]), pack_weights<BF16>(w[2], w[3]), pack_weights<BF16>(w[4], w[5]), pack_weights<BF16>(w[6], w[7])};
    l = product16<BF16>(ones16<BF16>(), p, l);
#pragma unroll
    for (int ct = 0; ct < kChannelTiles; ++ct) {
      const uint32_t pick = ct & 1 ? 0x07060302u : 0x05040100u;
      u32x4 vt;
#pragma unroll
      for (int x = 0; x < 4; ++x) vt[x] = __builtin_amdgcn_perm(v[2 * x + 1][ct >> 1], v[2 * x][ct >> 1], pick);
      o[ct] = product16<BF16>(vt, p, o[ct]);
    }
  }
  lsum += __shfl_xor(lsum, 16);
  lsum += __shfl_xor(lsum, 32);
  if (!live) return;
  const int64_t row = int64_t(span.first + i) * bt.num_kv_heads * a.rep + h * a.rep + r - i * a.rep;
  const float inv = l[0] == 0.f ? 0.f : 1.f / l[0];
  // channels of product ct: kChannelTiles * (4 j + x) + ct
  uint32_t* dst = reinterpret_cast<uint32_t*>(a.out + row * (2 * HD) + j * (HD / 2));
#pragma unroll
  for (int x = 0; x < 4; ++x)
#pragma unroll
    for (int y = 0; y < kChannelTiles / 2; ++y) dst[x * (kChannelTiles / 2) + y] = pack_out(o[2 * y][x] * inv, o[2 * y + 1][x] * inv, a.bf16);
  if (a.lse && j == 0) a.lse[row] = l[0] == 0.f ? -__builtin_inff() : (m + __builtin_amdgcn_logf(lsum)) * kLn2;
}

}  // namespace cocktail

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
  bool decode, tiles;
  int rows, row_tiles, workers;
  int64_t active;   // sequences that have queries at most
  size_t prefix_bytes, part_rows, bytes;
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
    int64_t workers = (units + 3) / 4;
    const int64_t fill = s.row_tiles <= 2 ? 2048 : 1024;
    workers = workers > fill ? fill : workers < 4 ? 4 : (workers + 3) / 4 * 4;
    s.workers = int(workers);
    s.prefix_bytes = (size_t(c->pages.num_seqs) + 1 + 63) / 64 * 256;
    s.part_rows = 2 * size_t(workers) * s.rows;
  }
  s.bytes = s.prefix_bytes + s.part_rows * (c->head_dim + 4) * sizeof(float) + 64;
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
  a.decode_rows = s.decode ? kDecodeRows : 0;
  char* w = static_cast<char*>(workspace);
  a.prefix = reinterpret_cast<int32_t*>(w);
  w += s.prefix_bytes;
  a.part_o = reinterpret_cast<float*>(w);
  w += s.part_rows * hd * sizeof(float);
  a.part_ml = reinterpret_cast<float*>(w);

  typedef void (*Kernel)(Kv16Attention);
  hipStream_t st = static_cast<hipStream_t>(stream);
  hipError_t e = hipSuccess;
  if (s.decode) {
    static const Kernel kernels[2][2][4] = {
        {{kv16_decode_kernel<64, false, 1>, kv16_decode_kernel<64, false, 2>, kv16_decode_kernel<64, false, 3>, kv16_decode_kernel<64, false, 4>},
         {kv16_decode_kernel<64, true, 1>, kv16_decode_kernel<64, true, 2>, kv16_decode_kernel<64, true, 3>, kv16_decode_kernel<64, true, 4>}},
        {{kv16_decode_kernel<128, false, 1>, kv16_decode_kernel<128, false, 2>, kv16_decode_kernel<128, false, 3>, kv16_decode_kernel<128, false, 4>},
         {kv16_decode_kernel<128, true, 1>, kv16_decode_kernel<128, true, 2>, kv16_decode_kernel<128, true, 3>, kv16_decode_kernel<128, true, 4>}}};
    e = launch_lds(kernels[hd == 128][a.bf16][s.row_tiles - 1], dim3(s.workers / kDecodeWaves), dim3(64 * kDecodeWaves), (a.batch.num_seqs + 1) * sizeof(int32_t), st, args);
  }
  if (e == hipSuccess && s.tiles) {
    static const Kernel kernels[2][2] = {{kv16_rows_kernel<64, false>, kv16_rows_kernel<64, true>}, {kv16_rows_kernel<128, false>, kv16_rows_kernel<128, true>}};
    const int64_t tiles = total * a.rep / 16 + s.active;
    e = launch(kernels[hd == 128][a.bf16], dim3(uint32_t(tiles * cache->num_kv_heads)), dim3(64), st, args);
  }
  if (e == hipSuccess && s.decode) {
    int most_new = kDecodeRows / a.rep < max_new ? kDecodeRows / a.rep : max_new;
    if (int64_t(cache->pages.num_seqs) * most_new > 4 * total) most_new = 0;
    const uint32_t most = uint32_t(most_new ? int64_t(cache->pages.num_seqs) * most_new : total) * num_q_heads;
    // states that a row has, about: many of them are read by many waves at a time, a few by one
    const int parts = int(s.workers / (s.active * cache->num_kv_heads));
    if (parts >= 16 && most <= 512)
      e = launch(hd == 128 ? merge_decode_kernel<Kv16Cost, 128, 16> : merge_decode_kernel<Kv16Cost, 64, 16>, dim3(most), dim3(1024), st, a, most_new);
    else if (parts >= 12 && most <= 2048)
      e = launch(hd == 128 ? merge_decode_kernel<Kv16Cost, 128, 4> : merge_decode_kernel<Kv16Cost, 64, 4>, dim3(most), dim3(256), st, a, most_new);
    else
      e = launch(hd == 128 ? merge_decode_kernel<Kv16Cost, 128, 1> : merge_decode_kernel<Kv16Cost, 64, 1>, dim3((most + 3) / 4), dim3(256), st, a, most_new);
  }
  if (e != hipSuccess) return fail(COCKTAIL_EHIP, "attention launch failed: %s", hipGetErrorString(e));
  return COCKTAIL_OK;
}
