// What the kernels of cocktail_fp4_attention share.
#pragma once
#include <type_traits>

#include "fp4_common.h"

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

struct Fp4Attention {
  Fp4Batch batch;
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
};

// A sequence as one kernel sees it: its rows (none if they are the other kernel's), tokens that the table holds, tokens before the new ones.  Query i
// sees tokens 0 .. past + i, as far as there are any.
struct Fp4Seq {
  int first, n, len, past;
};

__device__ __forceinline__ Fp4Seq decode_seq(const Fp4Attention& a, int b) {
  const Fp4Span s = fp4_span(a.batch, b);
  const int len = fp4_len(a.batch, b);
  return {s.first, s.count * a.rep <= a.decode_rows ? s.count : 0, fp4_held(a.batch, len), len - s.count};
}
__device__ __forceinline__ int seen_by(const Fp4Seq& s, int i) { return min(s.past + i + 1, s.len); }

// Operands of 16 query rows that a sequence needs in the decode kernel, its units of keys, and what they cost: the conversions of K and V
// once, and products and weights per operand, each about as long (8 x 16K, 1 .. 6 tokens of 8 heads: 55.6 us by operands alone, 47.4 by operands + 1,
// 49.4 by operands + 2).
__device__ __forceinline__ int decode_operands(const Fp4Attention& a, const Fp4Seq& s) { return (s.n * a.rep + 15) >> 4; }
__device__ __forceinline__ int decode_units(const Fp4Seq& s) { return s.n > 0 ? (s.len + kUnit - 1) / kUnit : 0; }
__device__ __forceinline__ int unit_cost(const Fp4Attention& a, const Fp4Seq& s) { return decode_operands(a, s) + 1; }
__device__ __forceinline__ int decode_cost(const Fp4Attention& a, const Fp4Seq& s) { return decode_units(s) * unit_cost(a, s); }

// A wave's share of the cost: not less than the dearest unit's, so that a segment has units in every share that lies between its first and its last.
__device__ __forceinline__ uint32_t cost_share(uint32_t cost, int workers) {
  const uint32_t n = (cost + uint32_t(workers) - 1) / uint32_t(workers);
  return n < 5 ? 5 : n;
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
__device__ __forceinline__ void write_merged(const Fp4Attention& a, const Merged<HD>& r, int64_t row, int lane) {
  const float inv = r.l == 0.f ? 0.f : 1.f / r.l;
  if constexpr (HD == 128) {
    reinterpret_cast<uint32_t*>(a.out)[row * 64 + lane] = pack_out(r.o[0] * inv, r.o[1] * inv, a.bf16);
  } else {
    reinterpret_cast<uint16_t*>(a.out)[row * 64 + lane] = uint16_t(pack_out(r.o[0] * inv, 0.f, a.bf16));
  }
  if (a.lse && lane == 0) a.lse[row] = r.l == 0.f ? -__builtin_inff() : (r.top + __builtin_amdgcn_logf(r.lsum)) * kLn2;
}

}  // namespace cocktail
