// Tile kernel of cocktail_fp4_attention: many query rows (new tokens x query heads of a kv head), a prompt or a part of one.
//
// Bound by the matrix cores and, close behind, by the exponentials of the softmax.  A workgroup takes 128 rows of one (sequence, kv head), 32 per
// wave, and walks over the keys 64 at a time: codes are loaded two steps ahead of their use, become fp16 once per workgroup on
// their way to LDS (K as rows of channels, V transposed, both as the operands of 32x32x16 products want them), and serve all waves.
// S^T = K Q^T leaves a lane with one query row and half the keys of a step, in the order in which O^T = V^T P^T takes them (the
// tokens of V lie in LDS in that order), so weights stay in their lanes.
#pragma once
#include "fp4_attention.h"

namespace cocktail {

constexpr int kTileWaves = 4;
constexpr int kTileRows = 32 * kTileWaves;

template <int HD>
struct Fp4TileLds {
  static constexpr int kKeyStride = HD + 8;          // halves; rows shift by four banks
  static constexpr int kChannelStride = kTileKeys + 8;
  _Float16 k[kTileKeys * kKeyStride];
  _Float16 v[HD * kChannelStride];
  int32_t ok[4];
};

__device__ __forceinline__ int tile_count(const Fp4Attention& a, const Fp4Span& s) {
  return s.count * a.rep > a.decode_rows ? (s.count * a.rep + kTileRows - 1) / kTileRows : 0;
}

template <int HD>
__global__ __launch_bounds__(64 * kTileWaves, 2) void fp4_tile_kernel(Fp4Attention a) {
  constexpr int kThreads = 64 * kTileWaves;
  constexpr int kSteps = HD / 16, kChannelTiles = HD / 32;
  constexpr int kItems = 2 * HD;                     // 16-byte pieces of 64 keys, of K and of V each
  __shared__ Fp4TileLds<HD> lds;
  __shared__ int32_t found[4], scratch[kTileWaves + 1];
  const Fp4Batch& bt = a.batch;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;

  // which rows: heads first, so that the heaviest tiles of all heads come first and the tiles of a head, which read the same keys, run on the same XCD
  const int h = blockIdx.x % bt.num_kv_heads;
  const int number = blockIdx.x / bt.num_kv_heads / a.splits, split = blockIdx.x / bt.num_kv_heads % a.splits;   // tile of the batch, part of its keys
  int run_tiles = 0;
  if (tid == 0) found[0] = -1;
  for (int base = 0; base < bt.num_seqs; base += kThreads) {
    const int b = base + tid;
    const Fp4Span s = b < bt.num_seqs ? fp4_span(bt, b) : Fp4Span{0, 0};
    const int v = tile_count(a, s);
    int x = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int y = __shfl_up(x, d);
      if (lane >= d) x += y;
    }
    __syncthreads();
    if (lane == 63) scratch[wave] = x;
    __syncthreads();
    int before = run_tiles;
    for (int w = 0; w < kTileWaves; ++w) {
      if (w < wave) before += scratch[w];
      run_tiles += scratch[w];
    }
    const int mine = before + x - v;
    if (number >= mine && number < mine + v) {
      found[0] = b;
      found[1] = v - 1 - (number - mine);   // the last rows of a sequence see most keys: first
    }
    if (run_tiles > number) break;
  }
  __syncthreads();
  const int b = __builtin_amdgcn_readfirstlane(found[0]);
  if (b < 0) return;
  const int tile = __builtin_amdgcn_readfirstlane(found[1]);
  const Fp4Span span = fp4_span(bt, b);
  const int n = span.count, rows = n * a.rep, len = fp4_len(bt, b);
  const int r0 = tile * kTileRows;
  const int last_row = (r0 + kTileRows < rows ? r0 + kTileRows : rows) - 1;
  int most = len - n + last_row / a.rep + 1;          // keys that the last row sees
  most = most < 0 ? 0 : most;
  const int steps = (most + kTileKeys - 1) / kTileKeys;
  const int k0 = int(int64_t(steps) * split / a.splits), k1 = int(int64_t(steps) * (split + 1) / a.splits);

  // the wave's rows
  const int row_lane = lane & 31, half = lane >> 5;
  const int r = r0 + wave * 32 + row_lane, i = r / a.rep;
  const bool live = r < rows;
  const int lim = live ? len - n + i + 1 : 0;
  const int wave_first = r0 + wave * 32, wave_last = wave_first + 31 < rows ? wave_first + 31 : rows - 1;
  const int wave_most = wave_first < rows ? len - n + wave_last / a.rep + 1 : 0;   // beyond: nothing to do for this wave
  const int wave_free = wave_first + 31 < rows ? len - n + wave_first / a.rep + 1 : 0;   // below: no masking
  h8 q[kSteps];
  float c = a.scale;
  {
    u32x4 raw[kSteps] = {};
    if (live) {
      const char* src = a.q + (span.first + i) * a.stride_t + (h * a.rep + r - i * a.rep) * a.stride_h + half * 16;
#pragma unroll
      for (int s = 0; s < kSteps; ++s) raw[s] = *reinterpret_cast<const u32x4*>(src + s * 32);
    }
    if (a.bf16) {
      float top = 0.f;
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
#pragma unroll
        for (int x = 0; x < 4; ++x) top = fmaxf(top, fmaxf(fabsf(bf_lo(raw[s][x])), fabsf(bf_hi(raw[s][x]))));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float f = row_factor(top), inv = 1.f / f;
      c *= f;
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
#pragma unroll
        for (int x = 0; x < 4; ++x) raw[s][x] = pack_halves(bf_lo(raw[s][x]) * inv, bf_hi(raw[s][x]) * inv);
    }
    c = fmaxf(c, 1.2e-38f);
#pragma unroll
    for (int s = 0; s < kSteps; ++s) q[s] = __builtin_bit_cast(h8, raw[s]);
  }

  // a thread's pieces of every 64 keys: of K token key_k, channels 32 g .. 32 g + 31; of V a quad of tokens, eight channels
  constexpr bool kBoth = kItems <= kThreads / 2 ? false : true;   // else the first half of the threads takes K, the second V
  const int item = kBoth ? tid : tid % kItems;
  const bool does_k = kBoth || tid < kItems, does_v = kBoth || tid >= kItems;
  const int key_k = item / (HD / 32), g = item % (HD / 32);
  const int quad = item & 15, piece = item >> 4;
  const int P = bt.page_size;
  const int64_t run = fp4_run_bytes(HD, P);
  const int32_t* table = bt.table + int64_t(b) * bt.table_stride;
  auto page_of = [&](int tok) -> int { return tok < len ? table[tok / P] : -1; };
  struct Raw {
    u32x4 k, v;
    uint32_t ks, vs;
    int ok;
  };
  auto load = [&](int step, int id_k, int id_v) {
    Raw x = {};
    x.ks = 127;
    x.vs = 0x7f7f7f7fu;
    const int tk = step * kTileKeys + key_k, tv = step * kTileKeys + quad * 4;
    if (does_k && uint32_t(id_k) < uint32_t(bt.num_pages) && tk < len) {
      const char* base = bt.pool + (int64_t(id_k) * bt.num_kv_heads + h) * run;
      const int at = tk % P;
      x.k = *reinterpret_cast<const u32x4*>(base + at * (HD / 2) + g * 16);
      x.ks = *reinterpret_cast<const uint8_t*>(base + P * HD + at * (HD / 32) + g);
      x.ok = 1;
    }
    if (does_v && uint32_t(id_v) < uint32_t(bt.num_pages) && tv < len) {
      const char* base = bt.pool + (int64_t(id_v) * bt.num_kv_heads + h) * run;
      const int at = tv % P;
      x.v = *reinterpret_cast<const u32x4*>(base + P * (HD / 2) + at * (HD / 2) + piece * 16);
      x.vs = *reinterpret_cast<const uint32_t*>(base + P * HD + P * (HD / 32) + at * (HD / 32) + (piece >> 2) * 4);
#pragma unroll
      for (int t = 1; t < 4; ++t)
        if (tv + t >= len) x.v[t] = 0, x.vs = (x.vs & ~(255u << (8 * t))) | 127u << (8 * t);
    }
    return x;
  };
  auto stage = [&](const Raw& x, int step) {
    if (does_k) {
      const float s = __builtin_bit_cast(float, x.ks << 23);
      u32x4* dst = reinterpret_cast<u32x4*>(lds.k + key_k * Fp4TileLds<HD>::kKeyStride + g * 32);
#pragma unroll
      for (int y = 0; y < 4; ++y) dst[y] = u32x4{fp4_pair<0>(x.k[y], s), fp4_pair<1>(x.k[y], s), fp4_pair<2>(x.k[y], s), fp4_pair<3>(x.k[y], s)};
      // pages hold multiples of 16 tokens; keys behind the last one are masked by their number
      if (g == 0 && key_k % 16 == 0) lds.ok[key_k / 16] = x.ok || step * kTileKeys + key_k >= len;
    }
    if (does_v) {
      // tokens of 16 in the order of quads 0, 2, 1, 3
      const int place = (quad & ~3) | ((quad & 1) << 1) | ((quad >> 1) & 1);
      _Float16* dst = lds.v + piece * 8 * Fp4TileLds<HD>::kChannelStride + place * 4;
      const float s0 = fp4_scale(x.vs, 0), s1 = fp4_scale(x.vs, 1), s2 = fp4_scale(x.vs, 2), s3 = fp4_scale(x.vs, 3);
      auto put = [&](auto byte_tag) {
        constexpr int B = decltype(byte_tag)::value;
        const uint32_t x0 = fp4_pair<B>(x.v[0], s0), x1 = fp4_pair<B>(x.v[1], s1), x2 = fp4_pair<B>(x.v[2], s2), x3 = fp4_pair<B>(x.v[3], s3);
        *reinterpret_cast<u32x2*>(dst + (2 * B) * Fp4TileLds<HD>::kChannelStride) =
            u32x2{__builtin_amdgcn_perm(x1, x0, 0x05040100), __builtin_amdgcn_perm(x3, x2, 0x05040100)};
        *reinterpret_cast<u32x2*>(dst + (2 * B + 1) * Fp4TileLds<HD>::kChannelStride) =
            u32x2{__builtin_amdgcn_perm(x1, x0, 0x07060302), __builtin_amdgcn_perm(x3, x2, 0x07060302)};
      };
      put(std::integral_constant<int, 0>{});
      put(std::integral_constant<int, 1>{});
      put(std::integral_constant<int, 2>{});
      put(std::integral_constant<int, 3>{});
    }
  };

  float m = kNoMax, lsum = 0.f;
  f32x16 o[kChannelTiles];
#pragma unroll
  for (int ct = 0; ct < kChannelTiles; ++ct) o[ct] = f32x16{};

  int id_k = -1, id_v = -1;
  Raw next = {};
  if (k0 < k1) {
    next = load(k0, page_of(k0 * kTileKeys + key_k), page_of(k0 * kTileKeys + quad * 4));
    id_k = page_of((k0 + 1) * kTileKeys + key_k);
    id_v = page_of((k0 + 1) * kTileKeys + quad * 4);
  }
  for (int step = k0; step < k1; ++step) {
    __syncthreads();   // the step before has been read
    stage(next, step);
    if (step + 1 < k1) {
      next = load(step + 1, id_k, id_v);
      id_k = page_of((step + 2) * kTileKeys + key_k);
      id_v = page_of((step + 2) * kTileKeys + quad * 4);
    }
    __syncthreads();
    const int tok0 = step * kTileKeys;
    if (tok0 >= wave_most) continue;   // (the whole wave)
    f32x16 s[2];
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      s[tt] = f32x16{};
      const _Float16* src = lds.k + (tt * 32 + row_lane) * Fp4TileLds<HD>::kKeyStride + half * 8;
#pragma unroll
      for (int st = 0; st < kSteps; ++st)
        s[tt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const h8*>(src + st * 16), q[st], s[tt], 0, 0, 0);
    }
    const int ok0 = lds.ok[0], ok1 = lds.ok[1], ok2 = lds.ok[2], ok3 = lds.ok[3];
    if (tok0 + kTileKeys > wave_free || !(ok0 && ok1 && ok2 && ok3)) {
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          const int tok = tok0 + tt * 32 + 8 * (x >> 2) + 4 * half + (x & 3);
          const int ok = tt == 0 ? (x < 8 ? ok0 : ok1) : (x < 8 ? ok2 : ok3);
          s[tt][x] = ok && tok < lim ? s[tt][x] : -__builtin_inff();
        }
    }
    float top = s[0][0];
#pragma unroll
    for (int x = 1; x < 32; ++x) top = fmaxf(top, s[x >> 4][x & 15]);
    top *= c;
    if (__any(top > m + kMaxSlack)) {
      top = fmaxf(top, __shfl_xor(top, 32));
      const float raised = fmaxf(m, top), alpha = __builtin_amdgcn_exp2f(m - raised);
      m = raised;
      lsum *= alpha;
#pragma unroll
      for (int ct = 0; ct < kChannelTiles; ++ct) o[ct] *= alpha;
    }
    h8 p[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      float w8[8];
#pragma unroll
      for (int x = 0; x < 8; ++x) w8[x] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u >> 1][(u & 1) * 8 + x], c, -m));
      lsum += ((w8[0] + w8[1]) + (w8[2] + w8[3])) + ((w8[4] + w8[5]) + (w8[6] + w8[7]));
      p[u] = __builtin_bit_cast(h8, u32x4{pack_halves(w8[0], w8[1]), pack_halves(w8[2], w8[3]), pack_halves(w8[4], w8[5]), pack_halves(w8[6], w8[7])});
    }
#pragma unroll
    for (int ct = 0; ct < kChannelTiles; ++ct) {
      const _Float16* src = lds.v + (ct * 32 + row_lane) * Fp4TileLds<HD>::kChannelStride + half * 8;
#pragma unroll
      for (int u = 0; u < 4; ++u)
        o[ct] = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const h8*>(src + u * 16), p[u], o[ct], 0, 0, 0);
    }
  }

  lsum += __shfl_xor(lsum, 32);
  if (!live) return;
  const int64_t row = int64_t(span.first + i) * bt.num_kv_heads * a.rep + h * a.rep + r - i * a.rep;
  if (a.splits == 1) {
    const float inv = lsum == 0.f ? 0.f : 1.f / lsum;
    char* dst = a.out + row * (2 * HD);
#pragma unroll
    for (int ct = 0; ct < kChannelTiles; ++ct)
#pragma unroll
      for (int y = 0; y < 4; ++y)
        *reinterpret_cast<u32x2*>(dst + 2 * (ct * 32 + 8 * y + 4 * half)) =
            u32x2{pack_out(o[ct][4 * y] * inv, o[ct][4 * y + 1] * inv, a.bf16), pack_out(o[ct][4 * y + 2] * inv, o[ct][4 * y + 3] * inv, a.bf16)};
    if (a.lse && half == 0) a.lse[row] = lsum == 0.f ? -__builtin_inff() : (m + __builtin_amdgcn_logf(lsum)) * kLn2;
    return;
  }
  const int64_t at_row = int64_t(split) * bt.total * bt.num_kv_heads * a.rep + row;
  float* dst = a.tile_o + at_row * HD;
#pragma unroll
  for (int ct = 0; ct < kChannelTiles; ++ct)
#pragma unroll
    for (int y = 0; y < 4; ++y)
      *reinterpret_cast<f32x4*>(dst + ct * 32 + 8 * y + 4 * half) = f32x4{o[ct][4 * y], o[ct][4 * y + 1], o[ct][4 * y + 2], o[ct][4 * y + 3]};
  if (half == 0) {
    float* ml = a.tile_ml + at_row * 3;
    ml[0] = m;
    ml[1] = lsum;
    ml[2] = lsum;
  }
}

}  // namespace cocktail
