// Decode kernel of cocktail_fp4_attention: up to 64 query rows (new tokens x query heads of a kv head) per (sequence, kv head).
//
// Bound by memory up to 16 rows: a key costs 2 * 17/32 D bytes and 4 D * rows operations.  Measured (averages): 128K tokens, 40 heads (713 MB) 114 us, 6.3 TB/s;
// eight sequences of 1 .. 128K, 8 kv heads, 4 query heads each (698 MB) 113 .. 119 us; with more rows by the conversions, exponentials and
// products: eight sequences of 9 .. 16K, 8 kv heads, 8 .. 48 rows (102 MB) 34 us.  What it takes to read at the rate of the memory:
//  * Work is cut by tokens, not by sequences: the units of 32 tokens of all (sequence, kv head) segments lie one behind the other, each as long as it
//    costs, and every wave takes those that begin in its share of that line, whatever the lengths are.  The numbering is made on the device from seq_lens, so that lengths can change
//    under a captured graph.  A segment inside one share is finished by its wave, the others leave a partial state per wave.
//  * A lane's operands are whole pieces of memory: of K, 16 tokens x D/4 channels (lane = token t, quarter j) are one operand of a 16x16x32
//    product S^T = K Q^T, the channels being taken in an order of the product's own (the same for Q); of V, lane (c, j) has channels
//    [8 c, 8 c + 8) of tokens 4 j .. 4 j + 3, which after a transposition of pairs are the operands of O^T = V^T P^T.
//    The result layout of S^T (lane: a query row, tokens 4 j + x) is the operand layout of P^T with tokens numbered accordingly: weights
//    never leave their lane.
//  * Codes become fp16 with one instruction per pair that applies the scale as well.
//  * The reference of the weights is only raised when a logit exceeds what it was made for by 2^4 (exact, the result does not depend on it), so that the
//    common step has no exchange between lanes at all.
#pragma once
#include "fp4_attention.h"

namespace cocktail {

// 16 tokens of one (sequence, kv head) as a lane holds them.
template <int HD>
struct Fp4Tile {
  u32x4 k;          // HD 64: the first half
  uint32_t k_scale;
  u32x4 v;
  uint32_t v_scale;
  int ok;           // wave-uniform: the page is one
};

// What lies where on the line of costs: with up to 64 sequences every wave has them in its lanes, otherwise the workgroup has what is before every
// sequence in LDS (pre[0 .. num_seqs]), for one kv head.
struct Fp4Line {
  Fp4Seq seq;        // of sequence `lane`
  int cost, before;
  uint32_t total;    // of all sequences and kv heads
};

__device__ __forceinline__ Fp4Line make_line(const Fp4Attention& a, int32_t* pre, int32_t* scratch) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Fp4Line r = {};
  int run = 0;
  if (a.batch.num_seqs <= 64) {
    if (lane < a.batch.num_seqs) {
      r.seq = decode_seq(a, lane);
      r.cost = decode_cost(a, r.seq);
    }
    const int upto = wave_prefix(r.cost);
    r.before = upto - r.cost;
    run = __builtin_amdgcn_readlane(upto, 63);
    if (blockIdx.x == 0 && wave == 0) {
      if (lane < a.batch.num_seqs) a.prefix[lane] = r.before;
      if (lane == 0) a.prefix[a.batch.num_seqs] = run;
    }
  } else {
    for (int base = 0; base < a.batch.num_seqs; base += 64 * kDecodeWaves) {
      const int b = base + threadIdx.x;
      const int v = b < a.batch.num_seqs ? decode_cost(a, decode_seq(a, b)) : 0;
      const int x = wave_prefix(v);
      __syncthreads();
      if (lane == 63) scratch[wave] = x;
      __syncthreads();
      int before = run;
      for (int w = 0; w < kDecodeWaves; ++w) {
        if (w < wave) before += scratch[w];
        run += scratch[w];
      }
      if (b < a.batch.num_seqs) pre[b] = before + x - v;
    }
    if (threadIdx.x == 0) pre[a.batch.num_seqs] = run;
    __syncthreads();
    if (blockIdx.x == 0)
      for (int b = threadIdx.x; b <= a.batch.num_seqs; b += 64 * kDecodeWaves) a.prefix[b] = pre[b];
  }
  r.total = uint32_t(run) * uint32_t(a.batch.num_kv_heads);
  return r;
}

__device__ __forceinline__ Fp4Seq of_lane(const Fp4Seq& s, int lane) {
  return {__builtin_amdgcn_readlane(s.first, lane), __builtin_amdgcn_readlane(s.n, lane), __builtin_amdgcn_readlane(s.len, lane),
          __builtin_amdgcn_readlane(s.past, lane)};
}

// The sequence at place u of the line: the last one that costs anything and has no more than u before it.
struct Fp4Place {
  int b, before, cost;   // cost of a kv head
  Fp4Seq seq;
};
__device__ __forceinline__ Fp4Place find_place(const Fp4Attention& a, const Fp4Line& line, const int32_t* pre, uint32_t u) {
  Fp4Place p;
  const uint32_t heads = a.batch.num_kv_heads;
  if (a.batch.num_seqs <= 64) {
    const uint64_t candidates = __ballot(line.cost > 0 && uint32_t(line.before) * heads <= u);
    p.b = 63 - __builtin_clzll(candidates);
    p.before = __builtin_amdgcn_readlane(line.before, p.b);
    p.cost = __builtin_amdgcn_readlane(line.cost, p.b);
    p.seq = of_lane(line.seq, p.b);
  } else {
    int b = 0, e = a.batch.num_seqs;
    while (e - b > 1) {
      const int m = (b + e) >> 1;
      if (uint32_t(pre[m]) * heads <= u) b = m;
      else e = m;
    }
    // (of sequences with the same before them the search ends at the last, which is the one that costs something)
    p.b = __builtin_amdgcn_readfirstlane(b);
    p.before = __builtin_amdgcn_readfirstlane(pre[p.b]);
    p.cost = __builtin_amdgcn_readfirstlane(pre[p.b + 1]) - p.before;
    p.seq = of_lane(decode_seq(a, p.b), 0);
  }
  return p;
}

// WHOLE: a workgroup of kWholeWaves waves has one segment and shares it out among them, their states are joined in LDS: one launch, for short contexts.
// Held to 128 registers, so that two of them run on a compute unit (1024 segments of 2048 tokens: 54.2 -> 47.4 us).  SPLIT: as many workgroups have a
// segment, each for its part of the channels of V.
constexpr int kWholeWaves = 8;

// The number-th sequence that has queries for this kernel, or -1; for a workgroup of kWholeWaves waves, `lds`: kWholeWaves + 1 words.
__device__ __forceinline__ int nth_active(const Fp4Attention& a, int number, int32_t* lds) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int run = 0;
  if (threadIdx.x == 0) lds[kWholeWaves] = -1;
  for (int base = 0; base < a.batch.num_seqs && run <= number; base += 64 * kWholeWaves) {
    const int b = base + int(threadIdx.x);
    const bool active = b < a.batch.num_seqs && decode_seq(a, b).n > 0;
    const uint64_t mask = __ballot(active);
    __syncthreads();
    if (lane == 0) lds[wave] = __builtin_popcountll(mask);
    __syncthreads();
    int before = run;
    for (int w = 0; w < kWholeWaves; ++w) {
      if (w < wave) before += lds[w];
      run += lds[w];
    }
    if (active && before + __builtin_popcountll(mask & ((uint64_t(1) << lane) - 1)) == number) lds[kWholeWaves] = b;
  }
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(lds[kWholeWaves]);
}

// The number-th longest of up to 64 sequences, for a workgroup of kWholeWaves waves: a lane has a sequence, a wave counts which of its share of them are
// longer.  Those without queries come last.
__device__ __forceinline__ int nth_longest(const Fp4Attention& a, int number, Fp4Seq* seq) {
  constexpr int kShare = 64 / kWholeWaves;
  __shared__ int counted[kWholeWaves][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Fp4Seq s = {};
  uint32_t key = 0;
  if (lane < a.batch.num_seqs) {
    s = decode_seq(a, lane);
    const uint32_t units = s.n > 0 ? decode_units(s) + 1 : 0, most = (1u << 25) - 1;
    key = (units < most ? units : most) << 6 | uint32_t(63 - lane);   // no two alike
  }
  int longer = 0, before = 0;
#pragma unroll
  for (int c = 0; c < kShare; ++c) longer += uint32_t(__builtin_amdgcn_readlane(int(key), wave * kShare + c)) > key ? 1 : 0;
  counted[wave][lane] = longer;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWholeWaves; ++w) before += counted[w][lane];
  const int b = __builtin_ctzll(__ballot(lane < a.batch.num_seqs && before == number));
  *seq = of_lane(s, b);
  return b;
}

template <int HD, int RT, bool WHOLE, int SPLIT = 1>
__global__ __launch_bounds__(64 * (WHOLE ? kWholeWaves : kDecodeWaves), WHOLE ? 4 : RT <= 2 ? 2 : 1) void fp4_decode_kernel(Fp4Attention a) {
  constexpr int kSteps = HD / 32;        // products per 16 tokens of S
  constexpr int kChannelTiles = HD / 16 / SPLIT;   // of a wave's output
  extern __shared__ int32_t pre[];
  __shared__ int32_t lds_words[kWholeWaves + 1];
  // three or four operands of queries do not fit the registers next to their sums: every lane reads its own from LDS
  constexpr bool kKeepQ = RT <= 2;
  // the normaliser is the sum of the weights as they were rounded, so that a row whose values are all alike is that value: a product with ones, which
  // adds up over the lanes too, or sums of a lane's own where four registers more per operand are not there
  constexpr bool kOnes = RT <= 2;
  __shared__ float lds_state[WHOLE ? 1 : kDecodeWaves][WHOLE ? 1 : 16][WHOLE ? 1 : HD + 4];
  __shared__ u32x4 lds_q[kKeepQ ? 1 : kDecodeWaves][kKeepQ ? 1 : RT][kKeepQ ? 1 : kSteps][kKeepQ ? 1 : 64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c16 = lane & 15, j = lane >> 4;
  const Fp4Batch& bt = a.batch;
  Fp4Line line = {};
  int w = 0;
  uint32_t u = 0, end = 1;
  bool stream = false;
  if constexpr (!WHOLE) {
    line = make_line(a, pre, lds_words);
    const uint32_t share = cost_share(line.total, a.workers);
    w = __builtin_amdgcn_readfirstlane(blockIdx.x * kDecodeWaves + (threadIdx.x >> 6));
    u = w * share;
    end = u + share < line.total ? u + share : line.total;
    if (u >= end) return;
    // read once and not again before hundreds of MB have passed: past the caches, which then read faster (128K, 40 heads: 130 -> 111 us); what
    // fits them is left to them (64 sequences of up to 4K, 8 heads, again and again: 38 us, and 42 past the caches).  With more than one
    // operand of queries the memory is not what is waited for.
    stream = RT == 1 && uint64_t(line.total) / 2 * (kUnit * 17 / 16 * HD) > kCachedBytes;
  }
  const int own_part = SPLIT > 1 ? int(blockIdx.x % SPLIT) : 0;
  const int P = bt.page_size;
  const int64_t run = fp4_run_bytes(HD, P);
  // byte offsets of a lane's pieces in 16 tokens
  const uint32_t off_k = c16 * (HD / 2) + j * (HD / 8);
  const uint32_t off_ks = uint32_t(P) * HD + c16 * (HD / 32) + (HD == 128 ? j : j >> 1);
  const uint32_t off_v = uint32_t(P) * (HD / 2) + j * (2 * HD) + (HD == 128 ? c16 : c16 >> 1) * 16;
  const uint32_t off_vs = uint32_t(P) * HD + uint32_t(P) * (HD / 32) + j * (HD / 8) + (HD == 128 ? c16 >> 2 : c16 >> 3) * 4;

  bool first_segment = true;
  while (u < end) {
    Fp4Place place;
    int h, u0, u1;
    if constexpr (WHOLE) {
      const int grid = gridDim.x / SPLIT;
      int at = blockIdx.x / SPLIT;
      if (bt.num_seqs <= 64 && grid > kComputeUnits) {
        // two workgroups to a compute unit: the longest segments first, then beside them the shortest, then the others (64 sequences of 512 ..
        // 4097 tokens, 8 heads: 41.7 -> 37.4 us; all of the same length 35.3 -> 35.6)
        const int second = grid < 2 * kComputeUnits ? grid : 2 * kComputeUnits;
        if (at >= kComputeUnits && at < second) at = kComputeUnits + second - 1 - at;
        const int number = at / bt.num_kv_heads;
        h = at - number * bt.num_kv_heads;
        place.b = nth_longest(a, number, &place.seq);
      } else {
        const int number = at / bt.num_kv_heads;
        h = at - number * bt.num_kv_heads;
        // more sequences than rows: the workgroups are for those that have any
        place.b = bt.num_seqs > bt.total ? nth_active(a, number, lds_words) : number;
        if (place.b < 0) return;
        place.seq = of_lane(decode_seq(a, place.b), 0);
      }
      if (place.seq.n == 0) return;
      const uint32_t units = decode_units(place.seq);
      u0 = units * wave / kWholeWaves;
      u1 = units * (wave + 1) / kWholeWaves;
      u = end;
    } else {
      place = find_place(a, line, pre, u);
    }
    const int b = place.b, n = place.seq.n, len = place.seq.len, rows = n * a.rep;
    const uint32_t operands = decode_operands(a, place.seq), per_unit = operands + 1;
    if constexpr (!WHOLE) {
      const uint32_t cost = place.cost, local = u - uint32_t(place.before) * uint32_t(bt.num_kv_heads);
      h = local / cost;
      const uint32_t c0 = local - uint32_t(h) * cost, c1 = end - u < cost - c0 ? c0 + (end - u) : cost;
      u += c1 - c0;
      // the units that begin in c0 .. c1 - 1
      u0 = (c0 + per_unit - 1) / per_unit, u1 = (c1 + per_unit - 1) / per_unit;
      if (u0 == u1) {
        first_segment = false;
        continue;
      }
    }

    // the queries: lane (row c16, quarter j) has the channels that its K pieces have
    u32x4 raw[RT][kSteps] = {};
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int r = rt * 16 + c16, i = r / a.rep;
      if (r < rows) {
        const u32x4* src = reinterpret_cast<const u32x4*>(a.q + (place.seq.first + i) * a.stride_t + (h * a.rep + r - i * a.rep) * a.stride_h + j * (HD / 2));
#pragma unroll
        for (int s = 0; s < kSteps; ++s) raw[rt][s] = src[s];
      }
    }

    // The tiles of the segment in order.  Every step loads two tiles and reads the table for two further on, whether they exist or not
    // (the last ones are then loaded again): with loads under a condition, the number of those in flight is not known when the code is made,
    // and every wait becomes one for all of them.
    const int32_t* table = bt.table + int64_t(b) * bt.table_stride;
    const int tiles = (len + 15) / 16;
    const int last_tile = 2 * u1 < tiles ? 2 * u1 - 1 : tiles - 1;
    const int tiles_per_page = P / 16;
    int tile = 2 * u0, col = tile / tiles_per_page, in_page = tile - col * tiles_per_page;   // of the table read
    auto next_tile = [&](int& id, int& at) {
      id = table_entry(table + col);
      at = in_page;
      const int more = tile < last_tile ? 1 : 0;
      tile += more;
      in_page += more;
      const bool turn = in_page == tiles_per_page;
      col += turn ? 1 : 0;
      in_page = turn ? 0 : in_page;
    };
    int id0, id1, at0, at1;   // of the next two tiles to load
    next_tile(id0, at0);
    next_tile(id1, at1);
    const char* head = bt.pool + h * run;
    const int64_t page_bytes = run * bt.num_kv_heads;
    auto load_tile = [&](auto policy, Fp4Tile<HD>& t, int id, int at) __attribute__((always_inline)) {
      constexpr int kPolicy = decltype(policy)::value;
      // a resource per page: the address is a base in scalar registers, an offset of the lane that never changes and one of the tile; a page
      // that is none has no bytes, and reads of it give zeros
      t.ok = uint32_t(id) < uint32_t(bt.num_pages);
      const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(head + (t.ok ? id : 0) * page_bytes), 0, t.ok ? int(run) : 0, 0x00020000);
      const int rows = at * (8 * HD), scales = at * (HD / 2);   // 16 tokens
      if constexpr (HD == 128) {
        t.k = __builtin_amdgcn_raw_buffer_load_b128(rs, off_k, rows, kPolicy);
      } else {
        const u32x2 half = __builtin_amdgcn_raw_buffer_load_b64(rs, off_k, rows, kPolicy);
        t.k = u32x4{half[0], half[1], 0, 0};
      }
      t.v = __builtin_amdgcn_raw_buffer_load_b128(rs, off_v, rows, kPolicy);
      t.k_scale = __builtin_amdgcn_raw_buffer_load_b8(rs, off_ks, scales, 0);
      t.v_scale = __builtin_amdgcn_raw_buffer_load_b32(rs, off_vs, scales, 0);
    };
    auto load_unit = [&](auto policy, Fp4Tile<HD>& ta, Fp4Tile<HD>& tb) __attribute__((always_inline)) {
      load_tile(policy, ta, id0, at0);
      load_tile(policy, tb, id1, at1);
      next_tile(id0, at0);
      next_tile(id1, at1);
    };
    Fp4Tile<HD> x0, x1, y0, y1;
    if (stream) load_unit(std::integral_constant<int, 2>{}, x0, x1);
    else load_unit(std::integral_constant<int, 0>{}, x0, x1);

    h8 q[kKeepQ ? RT : 1][kSteps];
    float c[RT], m[RT], lsum[RT];
    std::conditional_t<kOnes, f32x4, float> l[RT];
    f32x4 o[RT][kChannelTiles];
    int lim[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      c[rt] = a.scale;
      if (a.bf16) {
        float top = 0.f;
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
#pragma unroll
          for (int x = 0; x < 4; ++x) top = fmaxf(top, fmaxf(fabsf(bf_lo(raw[rt][s][x])), fabsf(bf_hi(raw[rt][s][x]))));
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float f = row_factor(top), inv = 1.f / f;
        c[rt] *= f;
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
#pragma unroll
          for (int x = 0; x < 4; ++x) raw[rt][s][x] = pack_halves(bf_lo(raw[rt][s][x]) * inv, bf_hi(raw[rt][s][x]) * inv);
      }
      c[rt] = fmaxf(c[rt], 1.2e-38f);
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        if constexpr (kKeepQ) q[rt][s] = __builtin_bit_cast(h8, raw[rt][s]);
        else lds_q[wave][rt][s][lane] = raw[rt][s];
      }
      const int r = rt * 16 + c16;
      lim[rt] = r < rows ? seen_by(place.seq, r / a.rep) : 0;
      m[rt] = kNoMax;
      lsum[rt] = 0.f;
      l[rt] = {};
#pragma unroll
      for (int ct = 0; ct < kChannelTiles; ++ct) o[rt][ct] = f32x4{};
    }
    const int free_below = seen_by(place.seq, 0);   // tokens that every query sees

    auto compute = [&](auto operands, Fp4Tile<HD>& ta, Fp4Tile<HD>& tb, int tok0) __attribute__((always_inline)) {
      constexpr int kLive = decltype(operands)::value;   // of the RT operands of queries
      // logits
      f32x4 s[kLive][2];
      {
        const float sa = __builtin_bit_cast(float, ta.k_scale << 23), sb = __builtin_bit_cast(float, tb.k_scale << 23);
#pragma unroll
        for (int rt = 0; rt < kLive; ++rt) s[rt][0] = s[rt][1] = f32x4{};
#pragma unroll
        for (int st = 0; st < kSteps; ++st) {
          const u32x4 wa = {fp4_pair<0>(ta.k[st], sa), fp4_pair<1>(ta.k[st], sa), fp4_pair<2>(ta.k[st], sa), fp4_pair<3>(ta.k[st], sa)};
          const u32x4 wb = {fp4_pair<0>(tb.k[st], sb), fp4_pair<1>(tb.k[st], sb), fp4_pair<2>(tb.k[st], sb), fp4_pair<3>(tb.k[st], sb)};
#pragma unroll
          for (int rt = 0; rt < kLive; ++rt) {
            h8 qq;
            if constexpr (kKeepQ) qq = q[rt][st];
            else qq = __builtin_bit_cast(h8, lds_q[wave][rt][st][lane]);
            s[rt][0] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, wa), qq, s[rt][0], 0, 0, 0);
            s[rt][1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, wb), qq, s[rt][1], 0, 0, 0);
          }
        }
      }
      // keys that a query does not see, and what lies in places that no token has been stored to
      if (tok0 + kUnit > free_below || !ta.ok || !tb.ok) {
        const int ka = tok0 + 4 * j, kb = ka + 16;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
#pragma unroll
          for (int rt = 0; rt < kLive; ++rt) {
            s[rt][0][x] = ta.ok && ka + x < lim[rt] ? s[rt][0][x] : -__builtin_inff();
            s[rt][1][x] = tb.ok && kb + x < lim[rt] ? s[rt][1][x] : -__builtin_inff();
          }
          if (!(ta.ok && ka + x < len)) ta.v[x] = 0, ta.v_scale = (ta.v_scale & ~(255u << (8 * x))) | 127u << (8 * x);
          if (!(tb.ok && kb + x < len)) tb.v[x] = 0, tb.v_scale = (tb.v_scale & ~(255u << (8 * x))) | 127u << (8 * x);
        }
      }
      // weights
      h8 p[kLive];
#pragma unroll
      for (int rt = 0; rt < kLive; ++rt) {
        float top = fmaxf(fmaxf(fmaxf(s[rt][0][0], s[rt][0][1]), fmaxf(s[rt][0][2], s[rt][0][3])),
                          fmaxf(fmaxf(s[rt][1][0], s[rt][1][1]), fmaxf(s[rt][1][2], s[rt][1][3]))) * c[rt];
        if (__any(top > m[rt] + (kShift + kSlack))) {
          top = fmaxf(top, __shfl_xor(top, 16));
          top = fmaxf(top, __shfl_xor(top, 32));
          const float raised = fmaxf(m[rt], top - kShift), alpha = __builtin_amdgcn_exp2f(m[rt] - raised);
          m[rt] = raised;
          lsum[rt] *= alpha;
          l[rt] *= alpha;
#pragma unroll
          for (int ct = 0; ct < kChannelTiles; ++ct) o[rt][ct] *= alpha;
        }
        float w8[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) w8[x] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[rt][x >> 2][x & 3], c[rt], -m[rt]));
        lsum[rt] += ((w8[0] + w8[1]) + (w8[2] + w8[3])) + ((w8[4] + w8[5]) + (w8[6] + w8[7]));
        const u32x4 words = {pack_halves(w8[0], w8[1]), pack_halves(w8[2], w8[3]), pack_halves(w8[4], w8[5]), pack_halves(w8[6], w8[7])};
        p[rt] = __builtin_bit_cast(h8, words);
        if constexpr (kOnes) {
          const _Float16 one = _Float16(1.f);
          l[rt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(h8{one, one, one, one, one, one, one, one}, p[rt], l[rt], 0, 0, 0);
        } else {
          l[rt] = add_rounded(words[3], add_rounded(words[2], add_rounded(words[1], add_rounded(words[0], l[rt]))));
        }
      }
      // weighted sums
      const float va0 = fp4_scale(ta.v_scale, 0), va1 = fp4_scale(ta.v_scale, 1), va2 = fp4_scale(ta.v_scale, 2), va3 = fp4_scale(ta.v_scale, 3);
      const float vb0 = fp4_scale(tb.v_scale, 0), vb1 = fp4_scale(tb.v_scale, 1), vb2 = fp4_scale(tb.v_scale, 2), vb3 = fp4_scale(tb.v_scale, 3);
      auto pair_of_channels = [&](auto byte_tag, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, uint32_t b2, uint32_t b3, int ct) __attribute__((always_inline)) {
        constexpr int B = decltype(byte_tag)::value;
        const uint32_t x0 = fp4_pair<B>(a0, va0), x1 = fp4_pair<B>(a1, va1), x2 = fp4_pair<B>(a2, va2), x3 = fp4_pair<B>(a3, va3);
        const uint32_t y0 = fp4_pair<B>(b0, vb0), y1 = fp4_pair<B>(b1, vb1), y2 = fp4_pair<B>(b2, vb2), y3 = fp4_pair<B>(b3, vb3);
        const u32x4 even = {__builtin_amdgcn_perm(x1, x0, 0x05040100), __builtin_amdgcn_perm(x3, x2, 0x05040100), __builtin_amdgcn_perm(y1, y0, 0x05040100),
                            __builtin_amdgcn_perm(y3, y2, 0x05040100)};
        const u32x4 odd = {__builtin_amdgcn_perm(x1, x0, 0x07060302), __builtin_amdgcn_perm(x3, x2, 0x07060302), __builtin_amdgcn_perm(y1, y0, 0x07060302),
                           __builtin_amdgcn_perm(y3, y2, 0x07060302)};
#pragma unroll
        for (int rt = 0; rt < kLive; ++rt) {
          o[rt][ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, even), p[rt], o[rt][ct], 0, 0, 0);
          o[rt][ct + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, odd), p[rt], o[rt][ct + 1], 0, 0, 0);
        }
      };
      uint32_t a0 = ta.v[0], a1 = ta.v[1], a2 = ta.v[2], a3 = ta.v[3], b0 = tb.v[0], b1 = tb.v[1], b2 = tb.v[2], b3 = tb.v[3];
      if constexpr (HD == 64 || SPLIT > 1) {
        // 64 channels: a lane has half a piece, channels 4 c .. 4 c + 3; and the workgroup's own of those
        const int sh = (HD == 64 ? (c16 & 1) * 16 : 0) + own_part * (4 * kChannelTiles);
        a0 >>= sh, a1 >>= sh, a2 >>= sh, a3 >>= sh, b0 >>= sh, b1 >>= sh, b2 >>= sh, b3 >>= sh;
      }
      pair_of_channels(std::integral_constant<int, 0>{}, a0, a1, a2, a3, b0, b1, b2, b3, 0);
      if constexpr (kChannelTiles > 2) pair_of_channels(std::integral_constant<int, 1>{}, a0, a1, a2, a3, b0, b1, b2, b3, 2);
      if constexpr (kChannelTiles > 4) {
        pair_of_channels(std::integral_constant<int, 2>{}, a0, a1, a2, a3, b0, b1, b2, b3, 4);
        pair_of_channels(std::integral_constant<int, 3>{}, a0, a1, a2, a3, b0, b1, b2, b3, 6);
      }
    };

    // the next unit is on its way while one is worked on
    auto walk = [&](auto policy, auto operands) __attribute__((always_inline)) {
      for (int k = u0;;) {
        load_unit(policy, y0, y1);
        compute(operands, x0, x1, k * kUnit);
        if (++k >= u1) break;
        load_unit(policy, x0, x1);
        compute(operands, y0, y1, k * kUnit);
        if (++k >= u1) break;
      }
    };
    if (WHOLE && u0 == u1) {
      // (a wave without keys has the state of none)
    } else if constexpr (WHOLE) {
      walk(std::integral_constant<int, 0>{}, std::integral_constant<int, RT>{});
    } else if constexpr (RT == 1) {
      if (stream) walk(std::integral_constant<int, 2>{}, std::integral_constant<int, 1>{});
      else walk(std::integral_constant<int, 0>{}, std::integral_constant<int, 1>{});
    } else {
      const std::integral_constant<int, 0> cached;
      if (operands == 1) walk(cached, std::integral_constant<int, 1>{});
      else if (RT == 2 || operands == 2) walk(cached, std::integral_constant<int, 2>{});
      else if (RT == 3 || operands == 3) walk(cached, std::integral_constant<int, (RT < 3 ? RT : 3)>{});
      else walk(cached, std::integral_constant<int, RT>{});
    }

    // whole segments are finished here, others leave their state: a wave has at most one that ends behind its share (or begins before it) at
    // each end, so two places per wave are enough
    if constexpr (WHOLE) {
      constexpr int kWidth = HD / SPLIT;
      __shared__ float states[kWholeWaves][16 * RT][kWidth + 4];   // sums, then (m, l, l unrounded)
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        float sum = lsum[rt];
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        float* dst = states[wave][rt * 16 + c16];
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
          for (int y = 0; y < kChannelTiles / 2; ++y)
            *reinterpret_cast<f32x2*>(dst + j * (kWidth / 4) + x * kChannelTiles + 2 * y) = f32x2{o[rt][2 * y][x], o[rt][2 * y + 1][x]};
        if (j == 0) dst[kWidth] = m[rt], dst[kWidth + 1] = l[rt][0], dst[kWidth + 2] = sum;
      }
      __syncthreads();
      // a wave joins every eighth row, a lane two neighbouring channels
      for (int r = wave; r < rows; r += kWholeWaves) {
        float top = kNoMax;
#pragma unroll
        for (int v = 0; v < kWholeWaves; ++v) top = fmaxf(top, states[v][r][kWidth]);
        float own_l = 0.f, own_lsum = 0.f, o0 = 0.f, o1 = 0.f;
        const int pair = lane < kWidth / 2 ? lane : 0;
#pragma unroll
        for (int v = 0; v < kWholeWaves; ++v) {
          const float* src = states[v][r];
          const float weight = __builtin_amdgcn_exp2f(src[kWidth] - top);
          own_l += weight * src[kWidth + 1];
          own_lsum += weight * src[kWidth + 2];
          const f32x2 v2 = *reinterpret_cast<const f32x2*>(src + 2 * pair);
          o0 += weight * v2[0];
          o1 += weight * v2[1];
        }
        const int i = r / a.rep;
        const int64_t row = int64_t(place.seq.first + i) * bt.num_kv_heads * a.rep + h * a.rep + r - i * a.rep;
        const float inv = own_l == 0.f ? 0.f : 1.f / own_l;
        const int channel = 2 * pair / kChannelTiles * (HD / 16) + own_part * kChannelTiles + 2 * pair % kChannelTiles;
        if (lane < kWidth / 2) reinterpret_cast<uint32_t*>(a.out)[(row * HD + channel) / 2] = pack_out(o0 * inv, o1 * inv, a.bf16);
        if (a.lse && lane == 0 && own_part == 0) a.lse[row] = own_l == 0.f ? -__builtin_inff() : (top + __builtin_amdgcn_logf(own_lsum)) * kLn2;
      }
      return;
    }
    const bool whole = u0 == 0 && u1 == int(decode_units(place.seq));
    const int64_t slot = 2 * int64_t(w) + (first_segment ? 0 : 1);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      float sum = lsum[rt];
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
      const int r = rt * 16 + c16;
      float lr;
      if constexpr (kOnes) {
        lr = l[rt][0];
      } else {
        lr = l[rt];
        lr += __shfl_xor(lr, 16);
        lr += __shfl_xor(lr, 32);
      }
      if (whole) {
        if (r >= rows) continue;
        const int i = r / a.rep;
        const int64_t row = int64_t(place.seq.first + i) * bt.num_kv_heads * a.rep + h * a.rep + r - i * a.rep;
        const float inv = lr == 0.f ? 0.f : 1.f / lr;
        char* dst = a.out + row * (2 * HD) + j * (HD / 2);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          if constexpr (HD == 128) {
            u32x4 v;
#pragma unroll
            for (int y = 0; y < 4; ++y) v[y] = pack_out(o[rt][2 * y][x] * inv, o[rt][2 * y + 1][x] * inv, a.bf16);
            *reinterpret_cast<u32x4*>(dst + 16 * x) = v;
          } else {
            u32x2 v;
#pragma unroll
            for (int y = 0; y < 2; ++y) v[y] = pack_out(o[rt][2 * y][x] * inv, o[rt][2 * y + 1][x] * inv, a.bf16);
            *reinterpret_cast<u32x2*>(dst + 8 * x) = v;
          }
        }
        if (a.lse && j == 0) a.lse[row] = lr == 0.f ? -__builtin_inff() : (m[rt] + __builtin_amdgcn_logf(sum)) * kLn2;
      } else {
        // through LDS, so that a store is a kilobyte of whole rows: stored from where the products leave it, sixteen bytes of a line at a time, a
        // state took as long as a unit or two (16 tokens of 4 heads behind 16K, 8 kv heads: 38.7 -> 33.7 us; 8 x 16K, 48 rows: 58 -> 54)
        if (rt * 16 >= rows) continue;
        float* own = lds_state[wave][c16] + j * (HD / 4);
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
          for (int y = 0; y < kChannelTiles / 4; ++y)
            *reinterpret_cast<f32x4*>(own + x * kChannelTiles + 4 * y) = f32x4{o[rt][4 * y][x], o[rt][4 * y + 1][x], o[rt][4 * y + 2][x], o[rt][4 * y + 3][x]};
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        constexpr int kLanes = HD / 4, kAtOnce = 64 / kLanes;   // lanes of a row, rows of a store
        float* dst = a.part_o + (slot * a.rows + rt * 16) * HD;
#pragma unroll
        for (int x = 0; x < 16 / kAtOnce; ++x) {
          const int row = x * kAtOnce + lane / kLanes, at = lane % kLanes * 4;
          const f32x4 v = *reinterpret_cast<const f32x4*>(lds_state[wave][row] + at);
          if (rt * 16 + row < rows) *reinterpret_cast<f32x4*>(dst + row * HD + at) = v;
        }
        __builtin_amdgcn_wave_barrier();
        if (j == 0 && r < rows) {
          float* ml = a.part_ml + (slot * a.rows + r) * 3;
          ml[0] = m[rt];
          ml[1] = lr;
          ml[2] = sum;
        }
      }
    }
    first_segment = false;
  }
}

}  // namespace cocktail
