// What the kernels of attention over paged caches share (cocktail_fp4_attention, cocktail_kv16_attention): rows and units of keys, how the work is cut,
// partial states and how they are joined.
#pragma once
#include <type_traits>

#include "paged_batch.h"

namespace cocktail {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// Weights are 2^(logit - reference) and become fp16.  The reference of a row is kShift below the largest logit that it was made for, so that weights
// lie in the upper part of fp16's range: from 2^-25 of that logit's weight on they are normal numbers, and what is smaller is off by 2^-36 of it at most, which
// a million keys of a long tail together do not show in a 16-bit result (with the reference at the largest logit it were 2^-25: the tail of 128K keys
// behind one that is 17 nats above them came out half as large again).  A reference that is kSlack too small is raised: weights up to 2^15.  The tile
// kernel, whose waves have 32 rows that all wait while one is raised, has 2^-21 and 2^-32 (prompts of 8190 and 4095 tokens: 749 us without a shift, 748 with 7,
// 760 with 8, 767 with 11).
constexpr float kNoMax = -3.0e38f;      // reference of a row that has seen no key
constexpr float kShift = 11.0f, kSlack = 4.0f, kTileShift = 7.0f;
constexpr int kUnit = 32;               // tokens that a wave of the decode kernel takes at a time
constexpr int kDecodeRows = 64;         // query rows (tokens x heads of a kv head) that the decode kernel serves at most
constexpr int kDecodeWaves = 4;         // waves per workgroup there
constexpr int kComputeUnits = 256;
constexpr int kTileKeys = 64;           // keys per step of the tile kernel
constexpr uint64_t kCachedBytes = 256u << 20;   // the last cache before the memory
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct PagedAttention {
  PagedBatch batch;
  const char* q;
  char* out;
  float* lse;
  int64_t stride_t, stride_h;   // of q, bytes
  int32_t rep, bf16;            // query heads per kv head
  float scale;                  // sm_scale * log2(e)
  int32_t rows;                 // most rows that a partial state of the decode kernel has: min(max_new * rep, kDecodeRows)
  int32_t workers;              // waves of the decode kernel
  int32_t decode_rows;          // sequences with at most so many rows are the decode kernel's, the others the tile kernel's
  int32_t splits;               // parts that the tile kernel cuts the keys of a row into
  int32_t* prefix;              // workspace: cost of the sequences before b, for one kv head [num_seqs + 1]
  float* part_ml;               // (m, l, l unrounded) of the partial states
  float* part_o;                // their weighted sums
  float* tile_ml;
  float* tile_o;
  int32_t joins;                // where COST::kJoins: workgroups of the decode kernel whose waves all have parts of one segment leave one state
};

// A sequence as one kernel sees it: its rows (none if they are the other kernel's), tokens that the table holds, tokens before the new ones.  Query i
// sees tokens 0 .. past + i, as far as there are any.
struct PagedSeq {
  int first, n, len, past;
};

__device__ __forceinline__ PagedSeq decode_seq(const PagedAttention& a, int b) {
  const PagedSpan s = paged_span(a.batch, b);
  const int len = paged_len(a.batch, b);
  return {s.first, s.count * a.rep <= a.decode_rows ? s.count : 0, paged_held(a.batch, len), len - s.count};
}
__device__ __forceinline__ int seen_by(const PagedSeq& s, int i) { return min(s.past + i + 1, s.len); }

// Operands of 16 query rows that a sequence needs in the decode kernel, and its units of keys.  What a unit costs is the cache's own: COST::unit(a, s), of
// kMost at most.
__device__ __forceinline__ int decode_operands(const PagedAttention& a, const PagedSeq& s) { return (s.n * a.rep + 15) >> 4; }
__device__ __forceinline__ int decode_units(const PagedSeq& s) { return s.n > 0 ? (s.len + kUnit - 1) / kUnit : 0; }
template <class COST>
__device__ __forceinline__ int decode_cost(const PagedAttention& a, const PagedSeq& s) { return decode_units(s) * COST::unit(a, s); }

// A wave's share of the cost: not less than the dearest unit's, so that a segment has units in every share that lies between its first and its last.
template <class COST>
__device__ __forceinline__ uint32_t cost_share(uint32_t cost, int workers) {
  const uint32_t n = (cost + uint32_t(workers) - 1) / uint32_t(workers);
  return n < COST::kMost ? COST::kMost : n;
}

// Whether all waves of a workgroup of the decode kernel have parts of the segment [begin, end) of the line and nothing else.
__device__ __forceinline__ bool workgroup_joins(uint32_t begin, uint32_t end, uint32_t group, uint32_t share) {
  const uint32_t all = kDecodeWaves * share;
  return group * all >= begin && (group + 1) * all <= end;
}

__device__ __forceinline__ uint32_t pack_halves(float lo, float hi) {
  const _Float16 a = _Float16(lo), b = _Float16(hi);
  return as_u32(h2{a, b});
}
__device__ __forceinline__ uint32_t pack_out(float lo, float hi, int bf16) {
  if (!bf16) return pack_halves(lo, hi);
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, b2{__bf16(lo), __bf16(hi)});
}
// Sum of two weights as they were rounded, and of what was there before.
__device__ __forceinline__ float add_rounded(uint32_t w, float sum) {
  const _Float16 one = _Float16(1.f);
  return __builtin_amdgcn_fdot2(as_h2(w), h2{one, one}, sum, false);
}
// Two bf16 in a word as floats.
__device__ __forceinline__ float bf_lo(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return __builtin_bit_cast(float, w & 0xffff0000u); }

// Power of two that brings a row of bf16 values, the largest of which is `top`, below 2 (the largest of all below 4, so that the reciprocal is a
// normal number); 1 for rows of zeros.
__device__ __forceinline__ float row_factor(float top) {
  const uint32_t e = __builtin_bit_cast(uint32_t, top) >> 23;
  return top == 0.f ? 1.f : __builtin_bit_cast(float, (e < 1u ? 1u : e > 253u ? 253u : e) << 23);
}

// A word of the page table through the scalar data path: the table is written by other launches only, and the address is wave-uniform.
__device__ __forceinline__ int table_entry(const int32_t* p) {
  return *reinterpret_cast<const __attribute__((address_space(4))) int32_t*>(reinterpret_cast<uint64_t>(p));
}

// A row's joined state: reference maximum, sums of the weights rounded and unrounded, a lane's channels.
template <int HD>
struct Merged {
  float top, l, lsum, o[HD / 64];
};
template <int HD>
__device__ __forceinline__ void write_merged(const PagedAttention& a, const Merged<HD>& r, int64_t row, int lane) {
  const float inv = r.l == 0.f ? 0.f : 1.f / r.l;
  if constexpr (HD == 128) {
    reinterpret_cast<uint32_t*>(a.out)[row * 64 + lane] = pack_out(r.o[0] * inv, r.o[1] * inv, a.bf16);
  } else {
    reinterpret_cast<uint16_t*>(a.out)[row * 64 + lane] = uint16_t(pack_out(r.o[0] * inv, 0.f, a.bf16));
  }
  if (a.lse && lane == 0) a.lse[row] = r.l == 0.f ? -__builtin_inff() : (r.top + __builtin_amdgcn_logf(r.lsum)) * kLn2;
}

// What lies where on the line of costs: with up to 64 sequences every wave has them in its lanes, otherwise the workgroup has what is before every
// sequence in LDS (pre[0 .. num_seqs]), for one kv head.
struct CostLine {
  PagedSeq seq;        // of sequence `lane`
  int cost, before;
  uint32_t total;    // of all sequences and kv heads
};

template <class COST>
__device__ __forceinline__ CostLine make_line(const PagedAttention& a, int32_t* pre, int32_t* scratch) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  CostLine r = {};
  int run = 0;
  if (a.batch.num_seqs <= 64) {
    if (lane < a.batch.num_seqs) {
      r.seq = decode_seq(a, lane);
      r.cost = decode_cost<COST>(a, r.seq);
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
      const int v = b < a.batch.num_seqs ? decode_cost<COST>(a, decode_seq(a, b)) : 0;
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

__device__ __forceinline__ PagedSeq of_lane(const PagedSeq& s, int lane) {
  return {__builtin_amdgcn_readlane(s.first, lane), __builtin_amdgcn_readlane(s.n, lane), __builtin_amdgcn_readlane(s.len, lane),
          __builtin_amdgcn_readlane(s.past, lane)};
}

// The sequence at place u of the line: the last one that costs anything and has no more than u before it.
struct CostPlace {
  int b, before, cost;   // cost of a kv head
  PagedSeq seq;
};
__device__ __forceinline__ CostPlace find_place(const PagedAttention& a, const CostLine& line, const int32_t* pre, uint32_t u) {
  CostPlace p;
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

constexpr int kWholeWaves = 8;          // waves that share a segment where contexts are short

// The number-th sequence that has queries for this kernel, or -1; for a workgroup of WAVES waves, `lds`: WAVES + 1 words.
template <int WAVES = kWholeWaves>
__device__ __forceinline__ int nth_active(const PagedAttention& a, int number, int32_t* lds) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int run = 0;
  if (threadIdx.x == 0) lds[WAVES] = -1;
  for (int base = 0; base < a.batch.num_seqs && run <= number; base += 64 * WAVES) {
    const int b = base + int(threadIdx.x);
    const bool active = b < a.batch.num_seqs && decode_seq(a, b).n > 0;
    const uint64_t mask = __ballot(active);
    __syncthreads();
    if (lane == 0) lds[wave] = __builtin_popcountll(mask);
    __syncthreads();
    int before = run;
    for (int w = 0; w < WAVES; ++w) {
      if (w < wave) before += lds[w];
      run += lds[w];
    }
    if (active && before + __builtin_popcountll(mask & ((uint64_t(1) << lane) - 1)) == number) lds[WAVES] = b;
  }
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(lds[WAVES]);
}

// The number-th longest of up to 64 sequences, for a workgroup of kWholeWaves waves: a lane has a sequence, a wave counts which of its share of them are
// longer.  Those without queries come last.
__device__ __forceinline__ int nth_longest(const PagedAttention& a, int number, PagedSeq* seq) {
  constexpr int kShare = 64 / kWholeWaves;
  __shared__ int counted[kWholeWaves][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  PagedSeq s = {};
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

// The sequence of new token t: the last one that does not start behind it (those before it with the same start are empty).
__device__ __forceinline__ int seq_of_row(const PagedBatch& bt, int t) {
  if (!bt.starts) return t / bt.uniform;
  int b = 0, e = bt.num_seqs;
  while (e - b > 1) {
    const int mid = (b + e) >> 1;
    if (bt.starts[mid] <= t) b = mid;
    else e = mid;
  }
  return b;
}

// Sum of a row's partial states: `parts` of them, the k-th at row slot(k) of the arrays.
// Wave `wave` of `waves` takes every waves-th; o: the lane's channels, l and lsum: whole sums (in every wave).
template <int HD, class Slot>
__device__ __forceinline__ Merged<HD> merge_parts(const float* ml, const float* po, Slot&& slot, int parts, int wave, int waves, int lane) {
  constexpr int kPer = HD / 64;
  Merged<HD> r = {};
  r.top = kNoMax;
  for (int k = lane; k < parts; k += 64) r.top = fmaxf(r.top, ml[slot(k) * 3]);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) r.top = fmaxf(r.top, __shfl_xor(r.top, d));
  for (int base = 0; base < parts; base += 64) {
    float w = 0.f;
    if (base + lane < parts) {
      const float* x = ml + slot(base + lane) * 3;
      w = __builtin_amdgcn_exp2f(x[0] - r.top);
      r.l += w * x[1];
      r.lsum += w * x[2];
    }
    const int n = parts - base < 64 ? parts - base : 64;
    // eight states at a time on their way; behind the last one it is the last one again, with no weight
    for (int k = wave; k < n; k += 8 * waves) {
      float x[8][kPer];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float* src = po + slot(base + min(k + i * waves, n - 1)) * HD + lane * kPer;
#pragma unroll
        for (int y = 0; y < kPer; ++y) x[i][y] = src[y];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int at = k + i * waves;
        const float wk = at < n ? __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), min(at, n - 1))) : 0.f;
#pragma unroll
        for (int y = 0; y < kPer; ++y) r.o[y] += at < n ? wk * x[i][y] : 0.f;
      }
    }
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    r.l += __shfl_xor(r.l, d);
    r.lsum += __shfl_xor(r.lsum, d);
  }
  return r;
}

// Rows of the decode kernel, one per (sequence, new token, query head): joins what the waves (or workgroups) of its segment left, if there were several, and
// writes rows without keys.  WAVES waves for a row, at least four to a workgroup.  Numbered by sequence, most_new tokens each, or, where most of those
// would have no token, by new token (most_new 0), which is looked for among the sequences.
template <class COST, int HD, int WAVES>
__global__ __launch_bounds__(64 * (WAVES < 4 ? 4 : WAVES)) void merge_decode_kernel(PagedAttention a, int most_new) {
  constexpr int kPer = HD / 64, kRows = WAVES < 4 ? 4 / WAVES : 1;
  __shared__ float o[WAVES][HD];
  const PagedBatch& bt = a.batch;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % WAVES;
  const uint32_t heads = bt.num_kv_heads * a.rep;
  const uint32_t number = blockIdx.x * kRows + (WAVES < 4 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / WAVES : 0);
  const uint32_t hq = number % heads, bi = number / heads;
  if (bi >= uint32_t(most_new ? bt.num_seqs * most_new : bt.total)) return;   // (kRows > 1 only, where nobody waits for anybody)
  const int b = most_new ? bi / uint32_t(most_new) : seq_of_row(bt, bi);
  const uint32_t before = a.prefix[b], total = a.prefix[bt.num_seqs];
  const PagedSeq s = decode_seq(a, b);
  const int i = most_new ? bi % uint32_t(most_new) : int(bi) - s.first;
  if (i < 0 || i >= s.n) return;
  const uint32_t h = hq / uint32_t(a.rep);
  const int64_t row = int64_t(s.first + i) * heads + hq;
  const uint32_t units = decode_units(s), per_unit = COST::unit(a, s);
  Merged<HD> r = {};
  if (units > 0) {
    // the waves that the segment's first and last unit belong to
    const uint32_t share = cost_share<COST>(total * uint32_t(bt.num_kv_heads), a.workers);
    const uint32_t u0 = before * uint32_t(bt.num_kv_heads) + h * units * per_unit, u1 = u0 + (units - 1) * per_unit;
    const uint32_t w0 = u0 / share, w1 = u1 / share;
    if (w0 == w1) return;   // its wave has finished it
    const int in_state = i * a.rep + int(hq - h * a.rep);
    const int64_t first = (2 * int64_t(w0) + (u0 == w0 * share ? 0 : 1)) * a.rows + in_state;
    if (COST::kJoins && a.joins) {
      // waves, then workgroups (workgroup_joins), then waves
      const uint32_t all = kDecodeWaves * share, from = w0 / kDecodeWaves, to = w1 / kDecodeWaves + 1;
      const uint32_t g0 = u0 == from * all ? from : from + 1, g1 = u0 + units * per_unit == to * all ? to : to - 1;
      const int groups = g0 < g1 ? int(g1 - g0) : 0;
      const int head = groups ? int(kDecodeWaves * g0 - w0) : int(w1 - w0) + 1, tail = groups ? int(w1 + 1 - kDecodeWaves * g1) : 0;
      auto slot = [&](int k) -> int64_t {
        const int of = k < head ? int(w0) + k : k < head + groups ? kDecodeWaves * (int(g0) + k - head) : kDecodeWaves * int(g1) + (k - head - groups);
        return k == 0 ? first : 2 * int64_t(of) * a.rows + in_state;
      };
      r = merge_parts<HD>(a.part_ml, a.part_o, slot, head + groups + tail, wave, WAVES, lane);
    } else {
      const int64_t second = 2 * (int64_t(w0) + 1) * a.rows + in_state, step = 2 * int64_t(a.rows);
      r = merge_parts<HD>(a.part_ml, a.part_o, [&](int k) -> int64_t { return k == 0 ? first : second + (k - 1) * step; }, int(w1 - w0) + 1, wave, WAVES, lane);
    }
  }
  if constexpr (WAVES > 1) {
    if (wave) {
#pragma unroll
      for (int x = 0; x < kPer; ++x) o[wave][lane * kPer + x] = r.o[x];
    }
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int v = 1; v < WAVES; ++v)
#pragma unroll
      for (int x = 0; x < kPer; ++x) r.o[x] += o[v][lane * kPer + x];
  }
  write_merged<HD>(a, r, row, lane);
}

// Rows of the tile kernel whose keys were cut: a wave per (new token, query head).
template <class COST, int HD>
__global__ __launch_bounds__(256) void merge_tiles_kernel(PagedAttention a) {
  const PagedBatch& bt = a.batch;
  const int lane = threadIdx.x & 63;
  const int heads = bt.num_kv_heads * a.rep;
  const int row = __builtin_amdgcn_readfirstlane(int(blockIdx.x * 4 + (threadIdx.x >> 6)));
  if (row >= bt.total * heads) return;
  const int t = row / heads, b = seq_of_row(bt, t);
  const PagedSpan s = paged_span(bt, b);
  // not the rows of a sequence with a bad range, or of the decode kernel
  if (t < s.first || t >= s.first + s.count || s.count * a.rep <= a.decode_rows) return;
  const int64_t step = int64_t(bt.total) * heads;
  write_merged<HD>(a, merge_parts<HD>(a.tile_ml, a.tile_o, [&](int k) -> int64_t { return row + k * step; }, a.splits, 0, 1, lane), row, lane);
}

}  // namespace cocktail
