// Tile kernel of cocktail_kv16_attention: many query rows (new tokens x query heads of a kv head), a prompt or a part of one.
//
// Bound by the matrix cores and, close behind, by the exponentials of the softmax.  A workgroup takes 128 or 256 rows of one (sequence, kv head), 32
// per wave, and walks over the keys 64 at a time; K and V are loaded a step or two ahead of their use and go to LDS as they are, rows of channels in
// pieces of sixteen bytes, and serve all waves.  What a load of the products' operands touches is in different banks: of K, the same piece of
// sixteen rows, which are a piece longer than their channels; of V, which the transposing load reads, 32 bytes of four rows twice, whose pieces lie
// in an order of the row's own.
// Measured (averages): 2048 tokens of 4 x 8 heads of 128 behind 30K 0.99 .. 1.03 ms by card (1.04 .. 1.08 PFLOP/s; a large library product of fp16 matrices reaches 1.30, at a
// lower clock: power is a limit of both), a prompt of 16384 tokens, 32 heads 1.97 ms (1.11, of the products that are not masked), two of 8190 and 4095 0.70 .. 0.74 (0.93 .. 0.99).
// S^T = K Q^T leaves a lane with one query row and half the keys of a step, in the order in which O^T = V^T P^T takes them (the transposing load
// picks the tokens in that order), so weights stay in their lanes.
#pragma once
#include "kv16_attention.h"

namespace cocktail {

// K in chunks of 32 keys, a ring of five.  A step begins with the logits of its first chunk, reads the next two and writes the fourth and the fifth behind
// it: the fifth takes the place of the first, which was read before the barrier that the step began with.  V of 64 keys, twice.
constexpr int kChunk = 32, kRing = 5;
constexpr float kSumLimit = 61440.f;   // of the weights of 16 keys that a lane has: their largest is a finite fp16 then (behind a new reference it is 16 * 2^7 at most)
template <int HD>
struct Kv16TileLds {
  u32x4 k[kRing][kChunk * (HD / 8 + 1)];   // rows shift by four banks
  u32x4 v[2][kTileKeys * HD / 8];
};

template <bool BF16>
__device__ __forceinline__ f32x16 product32(u32x4 a, u32x4 b, f32x16 c) {
  if constexpr (BF16) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
}

// Four rows of sixteen columns of 16 bits, eight bytes of them in each of sixteen lanes: lane i gets column i.
__device__ __forceinline__ u32x2 load_transposed(const char* p) {
  typedef int16_t s4 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) s4 lds_s4;
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(p)));
}

template <int WAVES>
__device__ __forceinline__ int tile_count(const PagedAttention& a, const PagedSpan& s) {
  return s.count * a.rep > a.decode_rows ? (s.count * a.rep + 32 * WAVES - 1) / (32 * WAVES) : 0;
}

template <int HD, bool BF16, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void kv16_tile_kernel(Kv16Attention args) {
  constexpr int kThreads = 64 * WAVES, kTileRows = 32 * WAVES;
  constexpr int kSteps = HD / 16, kChannelTiles = HD / 32;
  constexpr int kRowPieces = HD / 8;                 // sixteen bytes each
  __shared__ Kv16TileLds<HD> lds;
  __shared__ int32_t found[4], scratch[WAVES];
  const PagedAttention& a = args.p;
  const PagedBatch& bt = a.batch;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  // which rows: heads first, so that the heaviest tiles of all heads come first and the tiles of a head, which read the same keys, run on the same XCD
  const uint32_t heads = bt.num_kv_heads, splits = a.splits;
  const int h = blockIdx.x % heads;
  const int number = blockIdx.x / heads / splits, split = blockIdx.x / heads % splits;   // tile of the batch, part of its keys
  int b, tile, first, n, all;
  if (bt.num_seqs <= 64) {
    // every wave has all sequences in its lanes: one read of them, and nobody waits for anybody
    const PagedSpan s = lane < bt.num_seqs ? paged_span(bt, lane) : PagedSpan{0, 0};
    const int tokens = lane < bt.num_seqs ? paged_len(bt, lane) : 0;
    const int v = tile_count<WAVES>(a, s), upto = wave_prefix(v);
    const uint64_t mask = __ballot(number >= upto - v && number < upto);
    if (!mask) return;
    b = __builtin_ctzll(mask);
    tile = __builtin_amdgcn_readlane(upto, b) - 1 - number;   // the last rows of a sequence see most keys: first
    first = __builtin_amdgcn_readlane(s.first, b);
    n = __builtin_amdgcn_readlane(s.count, b);
    all = __builtin_amdgcn_readlane(tokens, b);
  } else {
    int run_tiles = 0;
    if (tid == 0) found[0] = -1;
    for (int base = 0; base < bt.num_seqs; base += kThreads) {
      const int mine = base + tid;
      const int v = mine < bt.num_seqs ? tile_count<WAVES>(a, paged_span(bt, mine)) : 0;
      const int x = wave_prefix(v);
      __syncthreads();
      if (lane == 63) scratch[wave] = x;
      __syncthreads();
      int upto = run_tiles + x;
      for (int w = 0; w < WAVES; ++w) {
        if (w < wave) upto += scratch[w];
        run_tiles += scratch[w];
      }
      if (number >= upto - v && number < upto) {
        found[0] = mine;
        found[1] = upto - 1 - number;
      }
      if (run_tiles > number) break;
    }
    __syncthreads();
    b = __builtin_amdgcn_readfirstlane(found[0]);
    if (b < 0) return;
    tile = __builtin_amdgcn_readfirstlane(found[1]);
    const PagedSpan span = paged_span(bt, b);
    first = __builtin_amdgcn_readfirstlane(span.first);
    n = __builtin_amdgcn_readfirstlane(span.count);
    all = __builtin_amdgcn_readfirstlane(paged_len(bt, b));
  }
  const int rows = n * a.rep, len = paged_held(bt, all);
  const PagedSeq seq = {first, n, len, all - n};
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

  // A thread has a piece of each of kPieces keys of every step; those of a wave lie in the same sixteen tokens, so that where they are is a scalar.
  constexpr int kPieces = 8 * HD / kThreads, kKeysAtOnce = kTileKeys / kPieces, kWaveKeys = 64 / kRowPieces;
  const int own_key = tid / kRowPieces, piece = tid % kRowPieces;   // of the first of them
  const int P = bt.page_size;
  const int64_t run = int64_t(P) * (2 * HD);
  const int64_t page_bytes = run * bt.num_kv_heads;
  const int64_t head = h * run;
  const uint32_t off = (own_key & 15) * (2 * HD) + piece * 16;       // inside sixteen tokens (kKeysAtOnce is a multiple of those)
  const int wave_tile = wave * kWaveKeys >> 4;
  // where the piece of key `own_key` goes: K of a key within a chunk, V of a key within a step
  auto place_k = [&](int key) { return (key & 31) * (kRowPieces + 1) + piece; };
  auto place_v = [&](int key) { return key * kRowPieces + (piece ^ 4 * (HD == 128 ? key & 3 : key >> 1 & 1)); };

  // Where the 16-token tiles of the keys are: a lane knows one of 64, sixteen steps, and a step takes its own from there with a few scalar instructions
  // (looked up a tile after the other by the scalar unit, they cost a tenth of the kernel's time).  The table is read sixteen steps ahead; behind the
  // last tile it is the last tile again, which is masked by its number.  V of a step is loaded a step after its K.
  const int32_t* table = bt.table + int64_t(b) * bt.table_stride;
  const int last_tile = len > 0 ? (len - 1) >> 4 : 0;
  const uint32_t tiles_per_page = P / 16;
  int next16 = 4 * k0 + lane, ahead_id = 0, ahead_at = 0;   // of the next sixteen steps
  auto look_ahead = [&]() __attribute__((always_inline)) {
    const uint32_t t = next16 < last_tile ? next16 : last_tile, col = t / tiles_per_page;
    ahead_id = table[col];
    ahead_at = int(t - col * tiles_per_page) * (32 * HD);
    next16 += 64;
  };
  uint32_t place_lo = 0, place_hi = 0;   // bytes from the head's run of the first page
  uint64_t bad_tiles = 0;
  int taken = 64;                        // tiles of these that steps have taken
  u32x4 raw_k[kPieces], raw_v[kPieces];
  int64_t from_v[kPieces];         // of the step whose K was loaded last
  int bad_k;                       // its tiles that lie on no page, a bit each
  auto load_k = [&]() __attribute__((always_inline)) {
    if (taken == 64) {
      const bool ok = uint32_t(ahead_id) < uint32_t(bt.num_pages);
      const int64_t place = (ok ? ahead_id : 0) * page_bytes + ahead_at;
      place_lo = uint32_t(place);
      place_hi = uint32_t(place >> 32);
      bad_tiles = ~__ballot(ok);
      taken = 0;
      look_ahead();
    }
    bad_k = int(bad_tiles >> taken) & 15;
#pragma unroll
    for (int x = 0; x < kPieces; ++x) {
      const int at = taken + (x * kKeysAtOnce >> 4) + wave_tile;
      from_v[x] = head + int64_t(uint64_t(uint32_t(__builtin_amdgcn_readlane(int(place_hi), at))) << 32 | uint32_t(__builtin_amdgcn_readlane(int(place_lo), at)));
      raw_k[x] = *reinterpret_cast<const u32x4*>(bt.pool + from_v[x] + off);
    }
    taken += 4;
  };
  auto load_v = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < kPieces; ++x) raw_v[x] = *reinterpret_cast<const u32x4*>(args.v_pool + from_v[x] + off);
  };
  // What lies in places that no token has been stored to must not be taken for numbers: weights of zero do not hide a NaN.  (Of K it does not
  // matter, logits are masked.)
  auto clean_v = [&](int step, int bad) __attribute__((always_inline)) {
    if (!bad && (step + 1) * kTileKeys <= len) return;
#pragma unroll
    for (int x = 0; x < kPieces; ++x) {
      const int key = own_key + x * kKeysAtOnce;
      if ((bad >> (key >> 4) & 1) || step * kTileKeys + key >= len) raw_v[x] = u32x4{};
    }
  };
  // (the chunk of a step that the piece's key is in: with eight waves and 64 channels it is the thread's, else the piece's)
  auto stage_k = [&](int x, int slot_first, int slot_second) __attribute__((always_inline)) {
    const int key = own_key + x * kKeysAtOnce;
    lds.k[key >> 5 ? slot_second : slot_first][place_k(key)] = raw_k[x];
  };
  auto stage_v = [&](int x, int buffer) __attribute__((always_inline)) { lds.v[buffer][place_v(own_key + x * kKeysAtOnce)] = raw_v[x]; };

  // the queries
  u32x4 q[kSteps] = {};
  if (live) {
    const char* src = a.q + (first + i) * a.stride_t + (h * a.rep + r - i * a.rep) * a.stride_h + half * 16;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) q[s] = *reinterpret_cast<const u32x4*>(src + s * 32);
  }
  const float c = fmaxf(a.scale, 1.2e-38f);

  // the normaliser is the sum of the weights before they are rounded
  float m = kNoMax, lsum = 0.f;
  f32x16 o[kChannelTiles];
#pragma unroll
  for (int ct = 0; ct < kChannelTiles; ++ct) o[ct] = f32x16{};

  // Operands: of K, lane (row, half) has piece 2 x + half of its row; of V, 32 channels of the four tokens 4 half + .. and of those eight behind them.
  const uint32_t base_k = row_lane * (2 * HD + 16) + half * 16;
  auto read_k = [&](const u32x4* chunk, int x) __attribute__((always_inline)) {
    return *reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(chunk) + base_k + x * 32);
  };
  const int token = lane >> 2 & 3, swizzle_v = HD == 128 ? token : token >> 1;
  const uint32_t base_v = (4 * half + token) * (2 * HD) + (lane >> 4 & 1) * 32 + (lane & 3) * 8;
  auto read_v = [&](const u32x4* rows_v, int ct, int group) __attribute__((always_inline)) {   // group: of sixteen tokens
    const char* p = reinterpret_cast<const char*>(rows_v) + base_v + (ct ^ swizzle_v) * 64 + group * (32 * HD);
    const u32x2 lo = load_transposed(p), hi = load_transposed(p + 16 * HD);
    return u32x4{lo[0], lo[1], hi[0], hi[1]};
  };

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

  // One half of a step, for 32 keys with logits `s`: the logits of the next 32 (`ahead`, from `chunk`), next to the second half of these' weights; then
  // these' products with V (from `rows_v`), next to the first half of the next ones' weights and to the putting away of what has been loaded (`put`,
  // kPieces times).  So both kinds of products have as many exponentials beside them.  The order is written down and kept: a product every few other
  // instructions, its operands read four products before.
  uint32_t w[8];                    // weights of the next products with V, those of keys 0 .. 15 from the half step before
  float first_sum = 0.f;            // of these
  auto weigh = [&](const f32x16& s, int y, float& sum) __attribute__((always_inline)) {
    const float a0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[y], c, -m)), a1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[y + 1], c, -m));
    sum += a0 + a1;
    w[y / 2] = pack_weights<BF16>(a0, a1);
  };
  auto half_step = [&](const f32x16& s, f32x16& ahead, const u32x4* chunk, const u32x4* rows_v, int next_tok, int next_bad, auto&& put) __attribute__((always_inline)) {
    constexpr int kLead = 4;
    constexpr int kProductsV = 2 * kChannelTiles;
    constexpr int kOrder = 0x4 | 0x10 | 0x20 | 0x40;   // scalar instructions and loads may move
    u32x4 kf[kSteps], vf[kProductsV];
    auto fetch_k = [&](int x) { kf[x] = read_k(chunk, x); };
    auto fetch_v = [&](int x) { vf[x] = read_v(rows_v, x % kChannelTiles, x / kChannelTiles); };
    ahead = f32x16{};
    float sum = first_sum;
#pragma unroll
    for (int x = 0; x < kLead; ++x) fetch_k(x);
    __builtin_amdgcn_sched_barrier(kOrder);
    constexpr int kEveryK = kSteps / 4, kEveryV = kProductsV / 4;   // products per pair of weights
#pragma unroll
    for (int x = 0; x < kSteps; ++x) {
      if (x + kLead < kSteps) fetch_k(x + kLead);
      else if (x + kLead - kSteps < kProductsV) fetch_v(x + kLead - kSteps);
      ahead = product32<BF16>(kf[x], q[x], ahead);
      if (x % kEveryK == kEveryK - 1) weigh(s, 8 + 2 * (x / kEveryK), sum);
      __builtin_amdgcn_sched_barrier(kOrder);
    }
    // Whether the reference is too small shows in the sum of the weights: then each of them was too large at most by that (the products have not
    // taken place, and the weights are computed again); no maximum is looked for before it is needed.
    if (__any(sum > kSumLimit)) {
      raise(s);
      sum = 0.f;
#pragma unroll
      for (int y = 0; y < 16; y += 2) weigh(s, y, sum);
    }
    lsum += sum;
    __builtin_amdgcn_s_setprio(1);   // the other wave of the SIMD is to be found beside its exponentials (1 %)
    const u32x4 p[2] = {u32x4{w[0], w[1], w[2], w[3]}, u32x4{w[4], w[5], w[6], w[7]}};
    mask(ahead, next_tok, next_bad);
    first_sum = 0.f;
#pragma unroll
    for (int x = 0; x < kProductsV; ++x) {
      if (x + kLead < kProductsV) fetch_v(x + kLead);
      o[x % kChannelTiles] = product32<BF16>(vf[x], p[x / kChannelTiles], o[x % kChannelTiles]);
      if (x % 2 == 0) put(x / 2);
      if (x % kEveryV == kEveryV - 1) weigh(ahead, 2 * (x / kEveryV), first_sum);
      __builtin_amdgcn_sched_barrier(kOrder);
    }
    __builtin_amdgcn_s_setprio(0);
  };

  if (k0 < k1) {
    // K of the first two steps and V of the first one into LDS, K of the third and V of the second on their way
    look_ahead();
    load_k();
    load_v();
    int bad0 = bad_k, bad1;         // of this step and of the next
    clean_v(k0, bad0);
#pragma unroll
    for (int x = 0; x < kPieces; ++x) stage_k(x, 0, 1), stage_v(x, 0);
    load_k();
    load_v();
    bad1 = bad_k;
#pragma unroll
    for (int x = 0; x < kPieces; ++x) stage_k(x, 2, 3);
    load_k();
    __syncthreads();
    const bool idle = wave_first >= rows;
    f32x16 s0, s1;
    if (!idle) {
      s0 = f32x16{};
#pragma unroll
      for (int x = 0; x < kSteps; ++x) s0 = product32<BF16>(read_k(lds.k[0], x), q[x], s0);
      mask(s0, k0 * kTileKeys, bad0 & 3);
#pragma unroll
      for (int y = 0; y < 8; y += 2) weigh(s0, y, first_sum);
    }
    __syncthreads();                // the first step writes into the chunk that these products have read
    int chunk = 0;                  // slot of this step's first chunk
    for (int step = k0; step < k1; ++step) {
      const int buffer = (step - k0) & 1;
      const int slot1 = chunk + 1 < kRing ? chunk + 1 : chunk + 1 - kRing, slot2 = chunk + 2 < kRing ? chunk + 2 : chunk + 2 - kRing;
      const int slot4 = chunk + 4 < kRing ? chunk + 4 : chunk + 4 - kRing, slot5 = chunk;
      clean_v(step + 1, bad1);
      if (!idle) {
        half_step(s0, s1, lds.k[slot1], lds.v[buffer], step * kTileKeys + kChunk, bad0 >> 2, [&](int x) { if (x < kPieces) stage_v(x, buffer ^ 1); });
        half_step(s1, s0, lds.k[slot2], lds.v[buffer] + kChunk * kRowPieces, (step + 1) * kTileKeys, bad1 & 3,
                  [&](int x) { if (x < kPieces) stage_k(x, slot4, slot5); });
      } else {
#pragma unroll
        for (int x = 0; x < kPieces; ++x) stage_v(x, buffer ^ 1), stage_k(x, slot4, slot5);
      }
      bad0 = bad1;
      bad1 = bad_k;
      load_v();
      load_k();
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
            u32x2{pack_out(o[ct][4 * y] * inv, o[ct][4 * y + 1] * inv, BF16), pack_out(o[ct][4 * y + 2] * inv, o[ct][4 * y + 3] * inv, BF16)};
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
