// Tile kernel of cocktail_fp4_attention: many query rows (new tokens x query heads of a kv head), a prompt or a part of one.
//
// Bound by the matrix cores and, close behind, by the exponentials of the softmax.  A workgroup takes 128 or 256 rows of one (sequence, kv head), 32
// per wave, and walks over the keys 64 at a time: codes are loaded a step or two ahead of their use, become fp16 once per workgroup on
// their way to LDS (K as rows of channels, V transposed, both as the operands of 32x32x16 products want them), and serve all waves.
// Measured: 2048 tokens of 4 x 8 heads of 128 behind 30K 1.08 .. 1.13 ms (940 .. 990 TFLOP/s; a large library product of fp16 matrices reaches 1132), two whole prompts of 8190 and
// 4095 tokens, 32 heads, 0.75 .. 0.77 ms (890 .. 920, of the products that are not masked).
// S^T = K Q^T leaves a lane with one query row and half the keys of a step, in the order in which O^T = V^T P^T takes them (the
// tokens of V lie in LDS in that order), so weights stay in their lanes.
#pragma once
#include "fp4_attention.h"

namespace cocktail {

// K in chunks of 32 keys, a ring of five.  A step begins with the logits of its first chunk, reads the next two and writes the fourth and the fifth behind
// it: the fifth takes the place of the first, which was read before the barrier that the step began with.  V of 64 keys, twice.
constexpr int kChunk = 32, kRing = 5;
constexpr float kSumLimit = 61440.f;   // of the weights of 16 keys that a lane has: their largest is a finite fp16 then (behind a new reference it is 16 * 2^7 at most)
template <int HD>
struct Fp4TileLds {
  static constexpr int kKeyStride = HD + 8;          // halves; rows shift by four banks
  static constexpr int kChannelStride = kTileKeys + 8;
  _Float16 k[kRing][kChunk * kKeyStride];
  _Float16 v[2][HD * kChannelStride];
};

template <int WAVES>
__device__ __forceinline__ int tile_count(const Fp4Attention& a, const Fp4Span& s) {
  return s.count * a.rep > a.decode_rows ? (s.count * a.rep + 32 * WAVES - 1) / (32 * WAVES) : 0;
}

// One of four values that are the same in all lanes, by the lane's own number.
__device__ __forceinline__ const char* pick(int k, const char* a, const char* b, const char* c, const char* d) {
  const uint64_t x = uint64_t(a), y = uint64_t(b), z = uint64_t(c), w = uint64_t(d);
  const uint32_t lo01 = (k & 1) ? uint32_t(y) : uint32_t(x), hi01 = (k & 1) ? uint32_t(y >> 32) : uint32_t(x >> 32);
  const uint32_t lo23 = (k & 1) ? uint32_t(w) : uint32_t(z), hi23 = (k & 1) ? uint32_t(w >> 32) : uint32_t(z >> 32);
  return reinterpret_cast<const char*>(uint64_t((k & 2) ? hi23 : hi01) << 32 | ((k & 2) ? lo23 : lo01));
}

template <int HD, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void fp4_tile_kernel(Fp4Attention a) {
  constexpr int kThreads = 64 * WAVES, kTileRows = 32 * WAVES;
  constexpr int kSteps = HD / 16, kChannelTiles = HD / 32;
  __shared__ Fp4TileLds<HD> lds;
  __shared__ int32_t found[4], scratch[WAVES];
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
    const int v = tile_count<WAVES>(a, s);
    const int x = wave_prefix(v);
    __syncthreads();
    if (lane == 63) scratch[wave] = x;
    __syncthreads();
    int before = run_tiles;
    for (int w = 0; w < WAVES; ++w) {
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
  const int rows = n * a.rep, all = __builtin_amdgcn_readfirstlane(fp4_len(bt, b)), len = fp4_held(bt, all);
  const Fp4Seq seq = {first, n, len, all - n};
  const int r0 = tile * kTileRows;
  const int last_row = (r0 + kTileRows < rows ? r0 + kTileRows : rows) - 1;
  int most = seen_by(seq, last_row / a.rep);          // keys that the last row sees
  most = most < 0 ? 0 : most;
  const uint32_t steps = (most + kTileKeys - 1) / kTileKeys;
  const int k0 = steps * uint32_t(split) / splits, k1 = steps * uint32_t(split + 1) / splits;   // (steps < 2^25, splits up to 64)

  // the wave's rows
  const int row_lane = lane & 31, half = lane >> 5;
  const int r = r0 + wave * 32 + row_lane, i = r / a.rep;
  const bool live = r < rows;
  const int lim = live ? seen_by(seq, i) : 0;
  const int wave_first = r0 + wave * 32;
  const int wave_free = wave_first + 31 < rows ? seen_by(seq, wave_first / a.rep) : 0;   // below: no masking

  // A thread's pieces of every 64 keys: kPieces words (of eight channels) of a key of K, and as many pairs of channels of a quad of tokens of V.
  constexpr int kPieces = HD * 8 / kThreads;
  constexpr int kParts = HD / 8 / kPieces;           // threads that share a key
  const int key = tid / kParts, part = tid % kParts, quad = tid & 15, v_part = tid >> 4;
  const int P = bt.page_size;
  const int64_t run = fp4_run_bytes(HD, P);
  const int64_t page_bytes = run * bt.num_kv_heads;
  const char* head = bt.pool + h * run;
  // offsets inside 16 tokens (in a page's run: 8 HD bytes of codes and HD / 2 of scales)
  const uint32_t off_k = (key & 15) * (HD / 2) + part * (4 * kPieces), off_ks = uint32_t(P) * HD + (key & 15) * (HD / 32) + (part * kPieces >> 2);
  const uint32_t off_v = uint32_t(P) * (HD / 2) + (quad & 3) * (2 * HD) + (v_part * kPieces >> 2) * 16;
  const uint32_t off_vs = uint32_t(P) * HD + uint32_t(P) * (HD / 32) + (quad & 3) * (HD / 8) + (v_part * kPieces >> 4) * 4;
  const int v_shift = kPieces == 4 ? 0 : 8 * (v_part * kPieces & 3);   // to the thread's bytes of a piece
  const int sub_k = key >> 4, sub_v = quad >> 2;

  // The 16-token tiles of the keys in order, as in the decode kernel: the table is read ahead of the loads, these ahead of their use, without
  // conditions (behind the last tile it is the last tile again, which is masked by its number).  V of a step is loaded a step after its K.
  const int32_t* table = bt.table + int64_t(b) * bt.table_stride;
  const int last_tile = len > 0 ? (len - 1) >> 4 : 0;
  const int tiles_per_page = P / 16;
  int next16 = 4 * k0, col = next16 / tiles_per_page, in_page = next16 - col * tiles_per_page;
  int id[4], at[4];
  auto next_tiles = [&]() __attribute__((always_inline)) {
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
  u32x4 raw_k, raw_v;
  uint32_t raw_ks, raw_vs;
  const char *v_rows, *v_scales;   // of the step whose K was loaded last
  int bad_k;                       // its tiles that lie on no page, a bit each
  auto load_k = [&]() __attribute__((always_inline)) {
    const char *rows_of[4], *scales_of[4];
    bad_k = 0;
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      const bool ok = uint32_t(id[y]) < uint32_t(bt.num_pages);
      bad_k |= ok ? 0 : 1 << y;
      const char* base = head + (ok ? id[y] : 0) * page_bytes;
      rows_of[y] = base + at[y] * (8 * HD);
      scales_of[y] = base + at[y] * (HD / 2);
    }
    const char* rows_k = pick(sub_k, rows_of[0], rows_of[1], rows_of[2], rows_of[3]) + off_k;
    if constexpr (kPieces == 4) {
      raw_k = *reinterpret_cast<const u32x4*>(rows_k);
    } else if constexpr (kPieces == 2) {
      const u32x2 x = *reinterpret_cast<const u32x2*>(rows_k);
      raw_k = u32x4{x[0], x[1], 0, 0};
    } else {
      raw_k = u32x4{*reinterpret_cast<const uint32_t*>(rows_k), 0, 0, 0};
    }
    raw_ks = *reinterpret_cast<const uint8_t*>(pick(sub_k, scales_of[0], scales_of[1], scales_of[2], scales_of[3]) + off_ks);
    v_rows = pick(sub_v, rows_of[0], rows_of[1], rows_of[2], rows_of[3]) + off_v;
    v_scales = pick(sub_v, scales_of[0], scales_of[1], scales_of[2], scales_of[3]) + off_vs;
  };
  auto load_v = [&]() __attribute__((always_inline)) {
    raw_v = *reinterpret_cast<const u32x4*>(v_rows);
    raw_vs = *reinterpret_cast<const uint32_t*>(v_scales);
  };
  // What lies in places that no token has been stored to must not be taken for numbers: weights of zero do not hide a NaN.  (Of K it does not
  // matter, logits are masked.)
  auto clean_v = [&](int step, int bad) __attribute__((always_inline)) {
    if (!bad && (step + 1) * kTileKeys <= len) return;
#pragma unroll
    for (int t = 0; t < 4; ++t)
      if ((bad >> sub_v & 1) || step * kTileKeys + quad * 4 + t >= len) raw_v[t] = 0, raw_vs = (raw_vs & ~(255u << (8 * t))) | 127u << (8 * t);
  };
  auto stage_k = [&](int piece, int slot) __attribute__((always_inline)) {
    const float s = __builtin_bit_cast(float, raw_ks << 23);
    u32x4* dst = reinterpret_cast<u32x4*>(lds.k[slot] + (key & 31) * Fp4TileLds<HD>::kKeyStride + part * (8 * kPieces));
    const uint32_t w = raw_k[piece];
    dst[piece] = u32x4{fp4_pair<0>(w, s), fp4_pair<1>(w, s), fp4_pair<2>(w, s), fp4_pair<3>(w, s)};
  };
  auto stage_v = [&](auto byte_tag, int buffer) __attribute__((always_inline)) {
    constexpr int B = decltype(byte_tag)::value;
    // tokens of 16 in the order of quads 0, 2, 1, 3
    const int place = (quad & ~3) | ((quad & 1) << 1) | ((quad >> 1) & 1);
    _Float16* dst = lds.v[buffer] + v_part * (2 * kPieces) * Fp4TileLds<HD>::kChannelStride + place * 4;
    const uint32_t x0 = fp4_pair<B>(raw_v[0] >> v_shift, fp4_scale(raw_vs, 0)), x1 = fp4_pair<B>(raw_v[1] >> v_shift, fp4_scale(raw_vs, 1));
    const uint32_t x2 = fp4_pair<B>(raw_v[2] >> v_shift, fp4_scale(raw_vs, 2)), x3 = fp4_pair<B>(raw_v[3] >> v_shift, fp4_scale(raw_vs, 3));
    *reinterpret_cast<u32x2*>(dst + (2 * B) * Fp4TileLds<HD>::kChannelStride) = u32x2{__builtin_amdgcn_perm(x1, x0, 0x05040100), __builtin_amdgcn_perm(x3, x2, 0x05040100)};
    *reinterpret_cast<u32x2*>(dst + (2 * B + 1) * Fp4TileLds<HD>::kChannelStride) =
        u32x2{__builtin_amdgcn_perm(x1, x0, 0x07060302), __builtin_amdgcn_perm(x3, x2, 0x07060302)};
  };
  auto stage_all_k = [&](int slot) __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < kPieces; ++x) stage_k(x, slot);
  };
  auto stage_v_piece = [&](int piece, int buffer) __attribute__((always_inline)) {
    if (piece == 0) stage_v(std::integral_constant<int, 0>{}, buffer);
    if constexpr (kPieces > 1) {
      if (piece == 1) stage_v(std::integral_constant<int, 1>{}, buffer);
    }
    if constexpr (kPieces > 2) {
      if (piece == 2) stage_v(std::integral_constant<int, 2>{}, buffer);
      if (piece == 3) stage_v(std::integral_constant<int, 3>{}, buffer);
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

  // the normaliser is the sum of the weights before they are rounded (that of the rounded ones as well: 3 % of the kernel's time, to take away an error
  // that is within the weights' own)
  float m = kNoMax, lsum = 0.f;
  f32x16 o[kChannelTiles];
#pragma unroll
  for (int ct = 0; ct < kChannelTiles; ++ct) o[ct] = f32x16{};

  // Logits of 32 keys that a row does not see.
  auto mask = [&](f32x16& s, int tok0, int bad) __attribute__((always_inline)) {   // bad: of the two 16-token tiles
    if (tok0 + kChunk > wave_free || bad) {
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        const int tok = tok0 + 8 * (x >> 2) + 4 * half + (x & 3);
        s[x] = !(bad >> (x >> 3) & 1) && tok < lim ? s[x] : -__builtin_inff();
      }
    }
  };
  // The reference of a row whose logits exceed it by too much is made for the largest of them.
  auto raise = [&](const f32x16& s) __attribute__((always_inline)) {
    float top = s[0];
#pragma unroll
    for (int x = 1; x < 16; ++x) top = fmaxf(top, s[x]);
    top *= c;
    top = fmaxf(top, __shfl_xor(top, 32));
    const float raised = fmaxf(m, top - kTileShift), alpha = __builtin_amdgcn_exp2f(m - raised);
    m = raised;
    lsum *= alpha;
#pragma unroll
    for (int ct = 0; ct < kChannelTiles; ++ct) o[ct] *= alpha;
  };

  // One half of a step: logits of the next 32 keys (`ahead`, from chunk `slot`), next to the weights of these (`s`); then these' products with V
  // (keys 32 * sub ... of `v`), next to the putting away of what has been loaded (`put`, kPieces times).  The order is written down
  // and kept: a product every few other instructions, its operands read four products before.
  auto half_step = [&](const f32x16& s, f32x16& ahead, const _Float16* k, const _Float16* v, auto&& put) __attribute__((always_inline)) {
    constexpr int kLead = 4;
    constexpr int kProductsV = 2 * kChannelTiles;
    constexpr int kOrder = 0x4 | 0x10 | 0x20 | 0x40;   // scalar instructions and loads may move
    const _Float16* ksrc = k + row_lane * Fp4TileLds<HD>::kKeyStride + half * 8;
    const _Float16* vsrc = v + row_lane * Fp4TileLds<HD>::kChannelStride + half * 8;
    h8 kf[kSteps], vf[kProductsV];
    auto read_k = [&](int x) { kf[x] = *reinterpret_cast<const h8*>(ksrc + x * 16); };
    auto read_v = [&](int x) { vf[x] = *reinterpret_cast<const h8*>(vsrc + (x % kChannelTiles) * 32 * Fp4TileLds<HD>::kChannelStride + (x / kChannelTiles) * 16); };
    ahead = f32x16{};
    uint32_t w[8];
    float sum = 0.f;
#pragma unroll
    for (int x = 0; x < kLead; ++x) read_k(x);
    __builtin_amdgcn_sched_barrier(kOrder);
    constexpr int kPer = 16 / kSteps;   // weights per product
#pragma unroll
    for (int x = 0; x < kSteps; ++x) {
      if (x + kLead < kSteps) read_k(x + kLead);
      else if (x + kLead - kSteps < kProductsV) read_v(x + kLead - kSteps);
      ahead = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf[x], q[x], ahead, 0, 0, 0);
#pragma unroll
      for (int y = x * kPer; y < (x + 1) * kPer; y += 2) {
        const float a0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[y], c, -m)), a1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[y + 1], c, -m));
        sum += a0 + a1;
        w[y / 2] = pack_halves(a0, a1);
      }
      __builtin_amdgcn_sched_barrier(kOrder);
    }
    // Whether the reference is too small shows in the sum of the weights: then each of them was too large at most by that (the products have not
    // taken place, and the weights are computed again); no maximum is looked for before it is needed.
    if (__any(sum > kSumLimit)) {
      raise(s);
      sum = 0.f;
#pragma unroll
      for (int y = 0; y < 16; y += 2) {
        const float a0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[y], c, -m)), a1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[y + 1], c, -m));
        sum += a0 + a1;
        w[y / 2] = pack_halves(a0, a1);
      }
    }
    lsum += sum;
    const h8 p[2] = {__builtin_bit_cast(h8, u32x4{w[0], w[1], w[2], w[3]}), __builtin_bit_cast(h8, u32x4{w[4], w[5], w[6], w[7]})};
#pragma unroll
    for (int x = 0; x < kProductsV; ++x) {
      if (x + kLead < kProductsV) read_v(x + kLead);
      o[x % kChannelTiles] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[x], p[x / kChannelTiles], o[x % kChannelTiles], 0, 0, 0);
      if (x % 2 == 0) put(x / 2);
      __builtin_amdgcn_sched_barrier(kOrder);
    }
  };

  if (k0 < k1) {
    // K of the first two steps and V of the first one into LDS, K of the third and V of the second on their way
    const int slot_of = key >> 5;   // which of a step's two chunks the thread's key is in
    next_tiles();
    load_k();
    next_tiles();
    load_v();
    int bad0 = bad_k, bad1;         // of this step and of the next
    clean_v(k0, bad0);
    stage_all_k(slot_of);
#pragma unroll
    for (int x = 0; x < kPieces; ++x) stage_v_piece(x, 0);
    load_k();
    next_tiles();
    load_v();
    bad1 = bad_k;
    stage_all_k(2 + slot_of);
    load_k();
    next_tiles();
    __syncthreads();
    const bool idle = wave_first >= rows;
    f32x16 s0, s1;
    if (!idle) {
      s0 = f32x16{};
      const _Float16* src = lds.k[0] + row_lane * Fp4TileLds<HD>::kKeyStride + half * 8;
#pragma unroll
      for (int x = 0; x < kSteps; ++x) s0 = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const h8*>(src + x * 16), q[x], s0, 0, 0, 0);
      mask(s0, k0 * kTileKeys, bad0 & 3);
    }
    __syncthreads();                // the first step writes into the chunk that these products have read
    int chunk = 0;                  // slot of this step's first chunk
    for (int step = k0; step < k1; ++step) {
      const int buffer = (step - k0) & 1;
      const int slot1 = chunk + 1 < kRing ? chunk + 1 : chunk + 1 - kRing, slot2 = chunk + 2 < kRing ? chunk + 2 : chunk + 2 - kRing;
      const int slot4 = chunk + 4 < kRing ? chunk + 4 : chunk + 4 - kRing, slot5 = chunk;
      const int write_slot = slot_of ? slot5 : slot4;
      clean_v(step + 1, bad1);
      if (!idle) {
        half_step(s0, s1, lds.k[slot1], lds.v[buffer], [&](int x) { if (x < kPieces) stage_v_piece(x, buffer ^ 1); });
        mask(s1, step * kTileKeys + kChunk, bad0 >> 2);
        half_step(s1, s0, lds.k[slot2], lds.v[buffer] + kChunk, [&](int x) { if (x < kPieces) stage_k(x, write_slot); });
      } else {
#pragma unroll
        for (int x = 0; x < kPieces; ++x) stage_v_piece(x, buffer ^ 1);
        stage_all_k(write_slot);
      }
      bad0 = bad1;
      bad1 = bad_k;
      load_v();
      load_k();
      next_tiles();
      if (!idle && step + 1 < k1) mask(s0, (step + 1) * kTileKeys, bad0 & 3);
      chunk = slot2;
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
