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
};

__device__ __forceinline__ int tile_count(const Fp4Attention& a, const Fp4Span& s) {
  return s.count * a.rep > a.decode_rows ? (s.count * a.rep + kTileRows - 1) / kTileRows : 0;
}

// One of four values that are the same in all lanes, by the lane's own number.
__device__ __forceinline__ const char* pick(int k, const char* a, const char* b, const char* c, const char* d) {
  const uint64_t x = uint64_t(a), y = uint64_t(b), z = uint64_t(c), w = uint64_t(d);
  const uint32_t lo01 = (k & 1) ? uint32_t(y) : uint32_t(x), hi01 = (k & 1) ? uint32_t(y >> 32) : uint32_t(x >> 32);
  const uint32_t lo23 = (k & 1) ? uint32_t(w) : uint32_t(z), hi23 = (k & 1) ? uint32_t(w >> 32) : uint32_t(z >> 32);
  return reinterpret_cast<const char*>(uint64_t((k & 2) ? hi23 : hi01) << 32 | ((k & 2) ? lo23 : lo01));
}

template <int HD>
__global__ __launch_bounds__(64 * kTileWaves, 2) void fp4_tile_kernel(Fp4Attention a) {
  constexpr int kThreads = 64 * kTileWaves;
  constexpr int kSteps = HD / 16, kChannelTiles = HD / 32;
  constexpr int kItems = 2 * HD;                     // 16-byte pieces of 64 keys, of K and of V each
  __shared__ Fp4TileLds<HD> buffers[2];
  __shared__ int32_t found[4], scratch[kTileWaves + 1];
  const Fp4Batch& bt = a.batch;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  // which rows: heads first, so that the heaviest tiles of all heads come first and the tiles of a head, which read the same keys, run on the same XCD
  const uint32_t heads = bt.num_kv_heads, splits = a.splits;
  const int h = blockIdx.x % heads;
  const int number = blockIdx.x / heads / splits, split = blockIdx.x / heads % splits;   // tile of the batch, part of its keys
  int run_tiles = 0;
  if (tid == 0) found[0] = -1;
  for (int base = 0; base < bt.num_seqs; base += kThreads) {
    const int b = base + tid;
    const Fp4Span s = b < bt.num_seqs ? fp4_span(bt, b) : Fp4Span{0, 0};
    const int v = tile_count(a, s);
    const int x = wave_prefix(v);
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
  const int first = __builtin_amdgcn_readfirstlane(span.first), n = __builtin_amdgcn_readfirstlane(span.count);
  const int rows = n * a.rep, len = __builtin_amdgcn_readfirstlane(fp4_len(bt, b));
  const int r0 = tile * kTileRows;
  const int last_row = (r0 + kTileRows < rows ? r0 + kTileRows : rows) - 1;
  int most = len - n + last_row / a.rep + 1;          // keys that the last row sees
  most = most < 0 ? 0 : most;
  const uint32_t steps = (most + kTileKeys - 1) / kTileKeys;
  const int k0 = steps * uint32_t(split) / splits, k1 = steps * uint32_t(split + 1) / splits;   // (steps < 2^25, splits up to 64)

  // the wave's rows
  const int row_lane = lane & 31, half = lane >> 5;
  const int r = r0 + wave * 32 + row_lane, i = r / a.rep;
  const bool live = r < rows;
  const int lim = live ? len - n + i + 1 : 0;
  const int wave_first = r0 + wave * 32, wave_last = wave_first + 31 < rows ? wave_first + 31 : rows - 1;
  const int wave_most = wave_first < rows ? len - n + wave_last / a.rep + 1 : 0;   // beyond: nothing to do for this wave
  const int wave_free = wave_first + 31 < rows ? len - n + wave_first / a.rep + 1 : 0;   // below: no masking

  // a thread's pieces of every 64 keys: of K token key_k, channels 32 g .. 32 g + 31; of V a quad of tokens, eight channels
  constexpr bool kBoth = kItems > kThreads / 2;      // else half of the threads takes K, the other half V
  const int item = kBoth ? tid : tid % kItems;
  const bool does_k = kBoth || tid < kItems, does_v = kBoth || tid >= kItems;   // the same for a wave
  const int key_k = item / (HD / 32), g = item % (HD / 32);
  const int quad = item & 15, piece = item >> 4;
  const int P = bt.page_size;
  const int64_t run = fp4_run_bytes(HD, P);
  const int64_t page_bytes = run * bt.num_kv_heads;
  const char* head = bt.pool + h * run;
  // offsets inside 16 tokens' codes, and from there to the scales less those of the tokens (in a page's run: 16 tokens are 8 HD bytes of codes
  // and HD / 2 of scales)
  const uint32_t off_k = (key_k & 15) * (HD / 2) + g * 16, off_ks = uint32_t(P) * HD + (key_k & 15) * (HD / 32) + g;
  const uint32_t off_v = uint32_t(P) * (HD / 2) + (quad & 3) * (2 * HD) + piece * 16;
  const uint32_t off_vs = uint32_t(P) * HD + uint32_t(P) * (HD / 32) + (quad & 3) * (HD / 8) + (piece >> 2) * 4;
  const int sub_k = key_k >> 4, sub_v = quad >> 2;

  // the 16-token tiles of the keys in order, as in the decode kernel: the table is read a step ahead of the loads, these a step ahead of their use,
  // without conditions (behind the last tile it is the last tile again, which is masked by its number)
  const int32_t* table = bt.table + int64_t(b) * bt.table_stride;
  const int last_tile = len > 0 ? (len - 1) >> 4 : 0;
  const int tiles_per_page = P / 16;
  int next16 = 4 * k0, col = next16 / tiles_per_page, in_page = next16 - col * tiles_per_page;
  int id[4], at[4];
  auto next_tiles = [&]() {
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      id[x] = table_entry(table + col);
      at[x] = in_page;
      const int more = next16 < last_tile ? 1 : 0;
      next16 += more;
      in_page += more;
      const bool turn = in_page == tiles_per_page;
      col += turn ? 1 : 0;
      in_page = turn ? 0 : in_page;
    }
  };
  struct Raw {
    u32x4 k, v;
    uint32_t ks, vs;
    int bad;   // of the four tiles, a bit each
  };
  auto load = [&]() {
    Raw x = {};
    const char *rows_of[4], *scales_of[4];
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      const bool ok = uint32_t(id[y]) < uint32_t(bt.num_pages);
      x.bad |= ok ? 0 : 1 << y;
      const char* base = head + (ok ? id[y] : 0) * page_bytes;
      rows_of[y] = base + at[y] * (8 * HD);
      scales_of[y] = base + at[y] * (HD / 2);
    }
    if (does_k) {
      x.k = *reinterpret_cast<const u32x4*>(pick(sub_k, rows_of[0], rows_of[1], rows_of[2], rows_of[3]) + off_k);
      x.ks = *reinterpret_cast<const uint8_t*>(pick(sub_k, scales_of[0], scales_of[1], scales_of[2], scales_of[3]) + off_ks);
    }
    if (does_v) {
      x.v = *reinterpret_cast<const u32x4*>(pick(sub_v, rows_of[0], rows_of[1], rows_of[2], rows_of[3]) + off_v);
      x.vs = *reinterpret_cast<const uint32_t*>(pick(sub_v, scales_of[0], scales_of[1], scales_of[2], scales_of[3]) + off_vs);
    }
    return x;
  };
  auto stage = [&](Raw& x, int step, Fp4TileLds<HD>& lds) {
    if (x.bad || (step + 1) * kTileKeys > len) {
      // what lies in places that no token has been stored to must not be taken for numbers: weights of zero do not hide a NaN.  (Of K it does
      // not matter, logits are masked.)
#pragma unroll
      for (int t = 0; t < 4; ++t)
        if ((x.bad >> sub_v & 1) || step * kTileKeys + quad * 4 + t >= len) x.v[t] = 0, x.vs = (x.vs & ~(255u << (8 * t))) | 127u << (8 * t);
    }
    if (does_k) {
      const float s = __builtin_bit_cast(float, x.ks << 23);
      u32x4* dst = reinterpret_cast<u32x4*>(lds.k + key_k * Fp4TileLds<HD>::kKeyStride + g * 32);
#pragma unroll
      for (int y = 0; y < 4; ++y) dst[y] = u32x4{fp4_pair<0>(x.k[y], s), fp4_pair<1>(x.k[y], s), fp4_pair<2>(x.k[y], s), fp4_pair<3>(x.k[y], s)};
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

  // the queries
  h8 q[kSteps];
  float c = a.scale;
  {
    u32x4 raw[kSteps] = {};
    if (live) {
      const char* src = a.q + (first + i) * a.stride_t + (h * a.rep + r - i * a.rep) * a.stride_h + half * 16;
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

  float m = kNoMax, lsum = 0.f;
  f32x16 o[kChannelTiles];
#pragma unroll
  for (int ct = 0; ct < kChannelTiles; ++ct) o[ct] = f32x16{};

  auto compute = [&](int step, int bad, const Fp4TileLds<HD>& lds) {
    const int tok0 = step * kTileKeys;
    f32x16 s[2];
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      s[tt] = f32x16{};
      const _Float16* src = lds.k + (tt * 32 + row_lane) * Fp4TileLds<HD>::kKeyStride + half * 8;
#pragma unroll
      for (int st = 0; st < kSteps; ++st)
        s[tt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const h8*>(src + st * 16), q[st], s[tt], 0, 0, 0);
    }
    if (tok0 + kTileKeys > wave_free || bad) {
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          const int tok = tok0 + tt * 32 + 8 * (x >> 2) + 4 * half + (x & 3);
          s[tt][x] = !(bad >> (2 * tt + (x >> 3)) & 1) && tok < lim ? s[tt][x] : -__builtin_inff();
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
  };

  // Two buffers: while the waves work on the keys in one, they put the next ones into the other; one barrier a step.
  if (k0 < k1) {
    next_tiles();
    Raw now = load();
    next_tiles();
    int bad = now.bad;
    stage(now, k0, buffers[0]);
    now = load();
    next_tiles();
    __syncthreads();
    for (int step = k0; step < k1; ++step) {
      const int at_buffer = (step - k0) & 1;
      const int bad_next = now.bad;
      if (step + 1 < k1) stage(now, step + 1, buffers[at_buffer ^ 1]);
      now = load();
      next_tiles();
      if (step * kTileKeys < wave_most) compute(step, bad, buffers[at_buffer]);
      bad = bad_next;
      __syncthreads();
    }
  }

  lsum += __shfl_xor(lsum, 32);
  if (!live) return;
  const int64_t row = int64_t(first + i) * bt.num_kv_heads * a.rep + h * a.rep + r - i * a.rep;
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
