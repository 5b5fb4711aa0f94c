// cocktail_beam_select / cocktail_beam_reorder: a step of beam search over the logits, and the reordering of what its hypotheses carry.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <type_traits>

#include "common.h"

namespace cocktail {

// The selection is two launches.  The first reads the logits once: a workgroup has a piece of a row, sums exponentials against a reference that is
// only raised when a logit exceeds it by far, and keeps the `keep` largest logits of the piece: a logit is compared with a bound that `keep` of the
// workgroup's are not below, made of the lanes' maxima, and only what reaches it goes into a buffer, which is sorted 64 at a time.  The second has a workgroup
// per request: it joins the pieces of every row to log sum exp, turns the pieces' candidates into values and selects among them.  All keys
// differ (a value, then the lower place first), so that the order in which candidates are met does not matter.
// Bound by memory with vector work close behind: 64 x 8 rows of 131072 in bf16 (134 MB) 38 us and 7, eight logits of a lane taking some 80 instructions; 8 x 8 rows of
// 65001 11 us and 7, four rows of 32000 in fp32 6.2 us and 5.9, which are launches, dependent loads and sorts of 64.
constexpr int kSelectWaves = 4;
constexpr int kMostKeep = COCKTAIL_MAX_KEEP;
constexpr int kPerLane = 8;              // logits that a lane takes at a time
static_assert(kMostKeep == 64, "a wave has a list of the best in its lanes");

// A float as an integer of the same order; 0 is below all numbers.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float from_ordered(uint32_t u) { return __builtin_bit_cast(float, u & 0x80000000u ? u & 0x7fffffffu : ~u); }
__device__ __forceinline__ uint64_t ordered(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  return u >> 63 ? ~u : u | uint64_t(1) << 63;
}
__device__ __forceinline__ double from_ordered(uint64_t u) { return __builtin_bit_cast(double, u >> 63 ? u & ~(uint64_t(1) << 63) : ~u); }

// Keys of the two launches: the larger one comes first; {} is none.
struct LogitKey {
  uint64_t x;   // ordered logit, then the complement of the token
};
struct ValueKey {
  uint64_t value;   // ordered value
  uint64_t place;   // complement of the row in the group, ordered logit (values of a row that binary64 cannot tell apart), complement of the token
};
__device__ __forceinline__ uint64_t value_place(int j, uint32_t logit, uint32_t token) {
  return uint64_t(63 - j) << 56 | uint64_t(logit) << 24 | (0xffffffu - token);
}
__device__ __forceinline__ bool before(uint32_t a, uint32_t b) { return a > b; }
__device__ __forceinline__ bool before(const LogitKey& a, const LogitKey& b) { return a.x > b.x; }
__device__ __forceinline__ bool before(const ValueKey& a, const ValueKey& b) { return a.value > b.value || (a.value == b.value && a.place > b.place); }

// What lane ^ X has.  Without a trip through shared memory: permutations within quads, mirrors and rotations of sixteen lanes, swaps of rows and of halves.
template <int X>
__device__ __forceinline__ uint32_t of_partner(uint32_t v) {
  auto dpp = [](uint32_t x, auto control) { return uint32_t(__builtin_amdgcn_update_dpp(0, int(x), decltype(control)::value, 0xf, 0xf, true)); };
  if constexpr (X == 1) return dpp(v, std::integral_constant<int, 0xB1>{});
  else if constexpr (X == 2) return dpp(v, std::integral_constant<int, 0x4E>{});
  else if constexpr (X == 4) return dpp(dpp(v, std::integral_constant<int, 0x141>{}), std::integral_constant<int, 0x1B>{});   // ^ 7, ^ 3
  else if constexpr (X == 8) return dpp(v, std::integral_constant<int, 0x128>{});
  else if constexpr (X == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return threadIdx.x & 16 ? r[0] : r[1];
  } else {
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return threadIdx.x & 32 ? r[0] : r[1];
  }
}
template <int X>
__device__ __forceinline__ uint64_t of_partner(uint64_t v) { return uint64_t(of_partner<X>(uint32_t(v >> 32))) << 32 | of_partner<X>(uint32_t(v)); }
template <int X>
__device__ __forceinline__ LogitKey of_partner(const LogitKey& k) { return {of_partner<X>(k.x)}; }
template <int X>
__device__ __forceinline__ ValueKey of_partner(const ValueKey& k) { return {of_partner<X>(k.value), of_partner<X>(k.place)}; }
__device__ __forceinline__ uint32_t of_lane(uint32_t v, int lane) { return uint32_t(__builtin_amdgcn_readlane(int(v), lane)); }
__device__ __forceinline__ uint64_t of_lane(uint64_t v, int lane) { return uint64_t(of_lane(uint32_t(v >> 32), lane)) << 32 | of_lane(uint32_t(v), lane); }
__device__ __forceinline__ LogitKey of_lane(const LogitKey& k, int lane) { return {of_lane(k.x, lane)}; }
__device__ __forceinline__ ValueKey of_lane(const ValueKey& k, int lane) { return {of_lane(k.value, lane), of_lane(k.place, lane)}; }

// The largest of the lanes' values, in all lanes.
__device__ __forceinline__ uint32_t wave_most(uint32_t v) {
  auto step = [&](uint32_t other) { v = other > v ? other : v; };
  step(of_partner<1>(v));
  step(of_partner<2>(v));
  step(of_partner<4>(v));
  step(of_partner<8>(v));
  step(of_partner<16>(v));
  step(of_partner<32>(v));
  return of_lane(v, 0);
}

// Steps of a bitonic network: the lane keeps the earlier or the later of its key and its partner's.  Pairs at distance STEP and below it, in
// blocks of SIZE that are brought into order and, every other one, into the opposite order; FALLING: which of the two the first block's is.
template <int SIZE, int STEP, bool FALLING, class Key>
__device__ __forceinline__ void merge_blocks(Key& k, int lane) {
  const Key other = of_partner<STEP>(k);
  const bool keep_first = (((lane & STEP) == 0) == (SIZE == 64 || (lane & SIZE) == 0)) == FALLING;
  if (before(other, k) == keep_first) k = other;
  if constexpr (STEP > 1) merge_blocks<SIZE, STEP / 2, FALLING>(k, lane);
}
// The keys of a wave in order: the first one in lane 0 (FALLING), or in lane 63.
template <bool FALLING, class Key>
__device__ __forceinline__ Key sorted(Key k, int lane) {
  merge_blocks<2, 1, true>(k, lane);
  merge_blocks<4, 2, true>(k, lane);
  merge_blocks<8, 4, true>(k, lane);
  merge_blocks<16, 8, true>(k, lane);
  merge_blocks<32, 16, true>(k, lane);
  merge_blocks<64, 32, FALLING>(k, lane);
  return k;
}
// The first 64, in order, of a list in order and one in the opposite order.
template <class Key>
__device__ __forceinline__ Key merged(Key a, const Key& b, int lane) {
  if (before(b, a)) a = b;
  merge_blocks<64, 32, true>(a, lane);
  return a;
}

// A wave's list of the best keys that it has met, and a buffer in LDS of those that may join it.
constexpr int kBuffer = 64 * (kPerLane + 1);
template <class Key>
struct Best {
  Key list, border;   // sorted over the lanes; the keep-th of them (only what comes before it can join)
  int count;          // in the buffer
  Key* buffer;
  int keep, lane;
  __device__ Best(Key* lds, int keep_, int lane_) : list{}, border{}, count(0), buffer(lds), keep(keep_), lane(lane_) {}
  // Offers a key per lane where `there`.  Room for 64 more is the caller's to see to (join_full).
  __device__ __forceinline__ void offer(const Key& k, bool there) {
    const uint64_t mask = __ballot(there);
    if (!mask) return;
    if (there) buffer[count + __builtin_amdgcn_mbcnt_hi(uint32_t(mask >> 32), __builtin_amdgcn_mbcnt_lo(uint32_t(mask), 0))] = k;
    count += __builtin_popcountll(mask);
  }
  __device__ __forceinline__ void join(int n) {   // the last n of the buffer
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    Key k = {};
    if (lane < n) k = buffer[count - n + lane];
    count -= n;
    list = merged(list, sorted<false>(k, lane), lane);
    border = of_lane(list, keep - 1);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  }
  __device__ __forceinline__ void join_full() {
    while (count >= 64) join(64);
  }
  __device__ __forceinline__ void join_all() {
    join_full();
    if (count) join(count);
  }
};

struct BeamSelect {
  const void* logits;
  int64_t stride_row;   // elements
  int32_t groups, beams, vocab, keep, pieces;
  const float* scores;
  const uint8_t* finished;
  int32_t eos;
  int32_t *source, *token;
  float* score;
  uint8_t* finished_out;
  double* sums;         // workspace: [rows][pieces] sum of exponentials
  LogitKey* keys;       // [rows][pieces][keep]
  float* tops;          // [rows][pieces] what the sum is against
};

// Whether a row has candidates that its logits say.
__device__ __forceinline__ bool reads_logits(const BeamSelect& a, int row) { return a.scores[row] > -__builtin_inff() && !(a.finished && a.finished[row]); }

// No number becomes none, an infinite one the largest.  (A maximum is the other operand where one is a quiet no-number, which the sum makes of a
// signalling one.)
__device__ __forceinline__ float clean_logit(float x) { return fminf(fmaxf(x + 0.f, -__builtin_inff()), FLT_MAX); }

// The largest of eight; what is no number is passed over, or comes out.  (The instruction itself: a maximum of the language quiets every operand first.)
__device__ __forceinline__ float most_of(const float* x) {
  auto max3 = [](float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
  };
  static_assert(kPerLane == 8, "");
  const float a = max3(x[0], x[1], x[2]), b = max3(x[3], x[4], x[5]), c = max3(x[6], x[7], a);
  return max3(b, c, c);
}

// Eight logits as they are in memory.
template <class T>
struct Logits {
  u32x4 w[sizeof(T) * kPerLane / 16];
  __device__ __forceinline__ float at(int i) const {
    if constexpr (sizeof(T) == 4) {
      const uint32_t word = w[i >> 2][i & 3];
      return __builtin_bit_cast(float, word);
    } else {
      const uint32_t word = w[0][i >> 1];
      return float(__builtin_bit_cast(T, uint16_t(i & 1 ? word >> 16 : word)));
    }
  }
};

// A wave's tile: eight logits a lane from a multiple of eight, counted from the row's first, those behind its end as none.  (Nothing is made of what a tile
// within the row brings, so that nobody waits for it here.)  Rows begin at any address of their elements, and the words of sixteen bytes with them: which
// logits are summed together must not depend on where a row lies, or equal rows would have different sums.  It costs nothing: both launches for 64 rows
// of 65001 in bf16 18.1 us, 17.6 with rows that begin at whole words, 17.8 either way with words counted from aligned addresses.
template <class T>
__device__ __forceinline__ void load_logits(const T* row, int vocab, int64_t tile, int lane, Logits<T>& x) {
  constexpr int kWords = sizeof(T) * kPerLane / 16;
  typedef u32x4 Words __attribute__((aligned(2)));   // (the hardware takes them from any address)
  const int64_t first = tile * (64 * kPerLane), at = first + lane * kPerLane;
  const T* src = row + at;
  if (first + 64 * kPerLane <= vocab) {
#pragma unroll
    for (int i = 0; i < kWords; ++i) x.w[i] = __builtin_nontemporal_load(reinterpret_cast<const Words*>(src) + i);
  } else {
#pragma unroll
    for (int i = 0; i < kPerLane; ++i) {
      const bool there = at + i < vocab;
      if constexpr (sizeof(T) == 4) {
        x.w[i >> 2][i & 3] = there ? __builtin_bit_cast(uint32_t, src[i]) : 0xff800000u;
      } else {
        const uint32_t v = there ? uint32_t(__builtin_bit_cast(uint16_t, src[i])) : __builtin_bit_cast(uint16_t, T(-__builtin_inff()));
        x.w[0][i >> 1] = i & 1 ? x.w[0][i >> 1] | v << 16 : v;
      }
    }
  }
}

constexpr float kLog2eBeam = 1.4426950408889634f;
constexpr float kSlackBeam = 16.f;   // by which a logit may exceed the reference: exponentials up to 2^23

template <class T>
__global__ __launch_bounds__(64 * kSelectWaves) void beam_pieces_kernel(BeamSelect a) {
  __shared__ LogitKey buffers[kSelectWaves][kBuffer];
  __shared__ double lds_sum[kSelectWaves];
  __shared__ float lds_top[kSelectWaves];
  __shared__ uint32_t lds_border;   // ordered value that `keep` logits of the workgroup's are not below
  if (threadIdx.x == 0) lds_border = 0;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = blockIdx.x / a.pieces, piece = blockIdx.x % a.pieces;
  const T* src = static_cast<const T*>(a.logits) + int64_t(row) * a.stride_row;
  // the piece's, then the wave's
  const int64_t tiles = (int64_t(a.vocab) + 64 * kPerLane - 1) / (64 * kPerLane);
  const int64_t tile0 = tiles * piece / a.pieces, tile1 = tiles * (piece + 1) / a.pieces;

  Best<LogitKey> best(buffers[wave], a.keep, lane);
  float ref = -FLT_MAX;          // of the wave's exponentials
  double sum = 0.0;              // of the lane's
  float lane_most = -__builtin_inff();
  float border = -FLT_MAX;       // logits below it are not wanted
  // two tiles are on their way while one is worked on
  Logits<T> next[2];
  int64_t tile = tile0 + wave;
  int done = 0;
#pragma unroll
  for (int d = 0; d < 2; ++d)
    if (tile + d * kSelectWaves < tile1) load_logits(src, a.vocab, tile + d * kSelectWaves, lane, next[d]);
  if (!reads_logits(a, row)) return;   // (behind the first loads, which it need not wait for)
  __syncthreads();
  auto step = [&](Logits<T>& own) __attribute__((always_inline)) {
    float x[kPerLane];
#pragma unroll
    for (int i = 0; i < kPerLane; ++i) x[i] = own.at(i);
    if (tile + 2 * kSelectWaves < tile1) load_logits(src, a.vocab, tile + 2 * kSelectWaves, lane, own);
    float most = most_of(x);
    auto raise = [&]() __attribute__((always_inline)) {
      const float raised = fmaxf(ref, fminf(from_ordered(wave_most(most == most && most > -__builtin_inff() ? ordered(most) : ordered(-FLT_MAX))), FLT_MAX));
      sum *= __builtin_amdgcn_exp2f((ref - raised) * kLog2eBeam);
      ref = raised;
    };
    auto exponentials = [&]() __attribute__((always_inline)) {
      float part = 0.f;
#pragma unroll
      for (int i = 0; i < kPerLane; ++i) part += __builtin_amdgcn_exp2f((x[i] - ref) * kLog2eBeam);
      return part;
    };
    if (__any(most > ref + kSlackBeam)) raise();
    float part = exponentials();
    if (__any(!(part < FLT_MAX))) {
      // logits that are no numbers or infinite
#pragma unroll
      for (int i = 0; i < kPerLane; ++i) x[i] = clean_logit(x[i]);
      most = most_of(x);
      raise();
      part = exponentials();
    }
    sum += part;
    lane_most = fmaxf(lane_most, most);
    // the bound: the keep-th of the lanes' maxima, after 1, 2, 4, 8 ... tiles, and what other waves found
    if ((done & (done + 1)) == 0) {
      const uint32_t mine = lane_most > -__builtin_inff() ? ordered(lane_most + 0.f) : 0;
      const uint32_t bound = of_lane(sorted<true>(mine, lane), a.keep - 1);
      if (bound) atomicMax(&lds_border, bound);
    }
    ++done;
    const uint32_t shared = lds_border;
    if (shared) border = fmaxf(border, from_ordered(shared));
    if (__any(most >= border)) {
      const int64_t at = (tile * 64 + lane) * kPerLane;
#pragma unroll
      for (int i = 0; i < kPerLane; ++i) {
        if (!__any(x[i] >= border)) continue;
        const LogitKey k = {uint64_t(ordered(x[i] + 0.f)) << 32 | uint32_t(~uint32_t(at + i))};   // (-0 as 0)
        best.offer(k, x[i] >= border && before(k, best.border));
      }
      if (best.count >= 64) {
        best.join_full();
        if (best.border.x) atomicMax(&lds_border, uint32_t(best.border.x >> 32));
      }
    }
  };
  while (tile < tile1) {
    step(next[0]);
    tile += kSelectWaves;
    if (tile >= tile1) break;
    step(next[1]);
    tile += kSelectWaves;
  }
  best.join_all();
  // the lanes' and the waves' states together
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
  if (lane == 0) lds_sum[wave] = sum, lds_top[wave] = ref;
  buffers[wave][lane] = best.list;
  __syncthreads();
  if (wave) return;
  LogitKey list = best.list;
  float top = ref;
  for (int w = 1; w < kSelectWaves; ++w) {
    list = merged(list, buffers[w][63 - lane], lane);
    const float other = lds_top[w], raised = fmaxf(top, other);
    sum = sum * __builtin_amdgcn_exp2f((top - raised) * kLog2eBeam) + lds_sum[w] * __builtin_amdgcn_exp2f((other - raised) * kLog2eBeam);
    top = raised;
  }
  const int64_t slot = int64_t(row) * a.pieces + piece;
  if (lane < a.keep) a.keys[slot * a.keep + lane] = list;
  if (lane == 0) a.sums[slot] = sum, a.tops[slot] = top;
}

// Sixteen waves: a row each (or several) for log sum exp, then 64 candidates each at a time, the best of all pieces first; the first wave joins what they kept.
constexpr int kJoinWaves = 16;
__global__ __launch_bounds__(64 * kJoinWaves) void beam_join_kernel(BeamSelect a) {
  __shared__ ValueKey kept[kJoinWaves * 64];
  __shared__ double log_sum[64], score_of[64];
  __shared__ float row_top[64];
  __shared__ uint8_t over[64];
  __shared__ unsigned long long lds_border;   // ordered value that `keep` candidates are not below
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int group = blockIdx.x, row0 = group * a.beams;
  const int lists = a.beams * a.pieces, all = lists * a.keep;
  if (threadIdx.x == 0) lds_border = 0;
  // the first candidates are on their way meanwhile
  LogitKey first_key = {};
  {
    const int i = int(threadIdx.x), rank = i / lists, at = i - rank * lists;
    if (i < all) first_key = a.keys[(int64_t(row0) * a.pieces + at) * a.keep + rank];   // (nothing, for rows that are not read: it is not used)
  }
  for (int j = wave; j < a.beams; j += kJoinWaves) {
    const int row = row0 + j;
    float top = -FLT_MAX;
    double sum = 0.0;
    const bool live = reads_logits(a, row);
    float next_top = -FLT_MAX;
    double next_sum = 0.0;
    if (lane < a.pieces) next_top = a.tops[int64_t(row) * a.pieces + lane], next_sum = a.sums[int64_t(row) * a.pieces + lane];
    if (live) {
      for (int p = lane; p < a.pieces; p += 64) {
        const int64_t slot = int64_t(row) * a.pieces + p;
        const float other = p < 64 ? next_top : a.tops[slot], raised = fmaxf(top, other);
        sum = sum * __builtin_amdgcn_exp2f((top - raised) * kLog2eBeam) + (p < 64 ? next_sum : a.sums[slot]) * __builtin_amdgcn_exp2f((other - raised) * kLog2eBeam);
        top = raised;
      }
      const float raised = from_ordered(wave_most(ordered(top)));
      sum *= __builtin_amdgcn_exp2f((top - raised) * kLog2eBeam);
      top = raised;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
    }
    if (lane == 0) {
      const bool ended = a.finished && a.finished[row];
      log_sum[j] = live ? log(sum) : 0.0;
      row_top[j] = top;
      score_of[j] = a.scores[row];
      over[j] = ended;
    }
  }
  __syncthreads();
  ValueKey list = {};
  for (int base = wave * 64; base < all; base += 64 * kJoinWaves) {
    // the best of every piece, then the second ones ...
    const int i = base + lane, rank = i / lists, at = i - rank * lists, j = i < all ? at / a.pieces : 0;
    const double score = score_of[j];
    ValueKey k = {};
    if (i < all && score > -__builtin_inf()) {
      if (over[j]) {
        if (rank == 0 && at == j * a.pieces) k = {ordered(score), value_place(j, 0, uint32_t(a.eos))};   // one candidate
      } else {
        const LogitKey x = base == wave * 64 ? first_key : a.keys[(int64_t(row0) * a.pieces + at) * a.keep + rank];
        const uint32_t logit = uint32_t(x.x >> 32);
        if (x.x) k = {ordered(score + ((double(from_ordered(logit)) - row_top[j]) - log_sum[j])), value_place(j, logit, ~uint32_t(x.x))};
      }
    }
    if (k.value < lds_border) k = {};
    if (!__any(k.value != 0)) continue;
    list = base == wave * 64 ? sorted<true>(k, lane) : merged(list, sorted<false>(k, lane), lane);
    const uint64_t bound = of_lane(list, a.keep - 1).value;
    if (bound && lane == 0) atomicMax(&lds_border, static_cast<unsigned long long>(bound));
  }
  // `keep` of every wave's
  if (lane < a.keep) kept[wave * a.keep + lane] = list;
  __syncthreads();
  if (wave) return;
  const int rest = a.keep * kJoinWaves;
  const uint64_t border = lds_border;
  list = lane < rest ? kept[lane] : ValueKey{};
  list = sorted<true>(list, lane);
  for (int base = 64; base < rest; base += 64) {
    ValueKey k = base + lane < rest ? kept[base + lane] : ValueKey{};
    if (k.value < border) k = {};
    if (__any(k.value != 0)) list = merged(list, sorted<false>(k, lane), lane);
  }
  if (lane >= a.keep) return;
  const bool there = list.value != 0;
  const int j = there ? 63 - int(list.place >> 56) : 0;
  const int v = 0xffffff - int(list.place & 0xffffffu);
  const int64_t at = int64_t(group) * a.keep + lane;
  a.source[at] = there ? row0 + j : -1;
  a.token[at] = there ? v : -1;
  a.score[at] = there ? float(from_ordered(list.value)) : -__builtin_inff();
  if (a.finished_out) a.finished_out[at] = there && (over[j] || v == a.eos) ? 1 : 0;
}

// ---- reordering ----------------------------------------------------------------------------------------------------------------

struct BeamStates {
  const char* from[COCKTAIL_MAX_STATES];
  char* to[COCKTAIL_MAX_STATES];
  int64_t row_bytes[COCKTAIL_MAX_STATES];
  int32_t num_states, rows;
};

__device__ __forceinline__ int beam_source(const int32_t* source, int row, int rows) {
  const int s = source[row];
  return s >= 0 && s < rows ? s : row;
}

// Rows into other memory: a workgroup has 4096 bytes of a row of a state.
constexpr int kCopyBytes = 4096;
template <class Word>
__device__ __forceinline__ void copy_words(char* to, const char* from, int bytes) {
  for (int i = threadIdx.x * int(sizeof(Word)); i < bytes; i += 256 * int(sizeof(Word))) *reinterpret_cast<Word*>(to + i) = *reinterpret_cast<const Word*>(from + i);
}
__device__ __forceinline__ int alignment(uint64_t bits) { return bits & 3 ? 1 : bits & 15 ? 4 : 16; }

__global__ __launch_bounds__(256) void beam_copy_kernel(const int32_t* source, BeamStates s) {
  const int row = blockIdx.y, of = source[row];
  if (of < 0 || of >= s.rows) return;
  int64_t chunk = blockIdx.x;
  for (int i = 0; i < s.num_states; ++i) {
    if (s.from[i] == s.to[i]) continue;
    const int64_t bytes = s.row_bytes[i], chunks = (bytes + kCopyBytes - 1) / kCopyBytes;
    if (chunk >= chunks) {
      chunk -= chunks;
      continue;
    }
    const int64_t at = chunk * kCopyBytes;
    const int n = int(bytes - at < kCopyBytes ? bytes - at : kCopyBytes);
    char* to = s.to[i] + row * bytes + at;
    const char* from = s.from[i] + of * bytes + at;
    const int align = alignment(reinterpret_cast<uintptr_t>(s.to[i]) | reinterpret_cast<uintptr_t>(s.from[i]) | uint64_t(bytes));
    if (align == 16) copy_words<u32x4>(to, from, n);
    else if (align == 4) copy_words<uint32_t>(to, from, n);
    else copy_words<uint8_t>(to, from, n);
    return;
  }
}

// Rows in place: a workgroup has a column of a state, all rows of it, which are read before any is written.
constexpr int kPlaceBytes = 65536;   // of a column, in LDS
template <class Word>
__device__ __forceinline__ void permute_words(const int32_t* source, char* state, int rows, int64_t row_bytes, int64_t at, int width, char* lds) {
  const int words = width / int(sizeof(Word)), all = rows * words;
  Word* held = reinterpret_cast<Word*>(lds);
  for (int i = threadIdx.x; i < all; i += 256) {
    const int row = i / words, w = i - row * words, of = beam_source(source, row, rows);
    if (of != row) held[i] = *reinterpret_cast<const Word*>(state + of * row_bytes + at + w * int(sizeof(Word)));
  }
  __syncthreads();
  for (int i = threadIdx.x; i < all; i += 256) {
    const int row = i / words, w = i - row * words;
    if (beam_source(source, row, rows) != row) *reinterpret_cast<Word*>(state + row * row_bytes + at + w * int(sizeof(Word))) = held[i];
  }
}

__host__ __device__ inline int column_bytes(int rows) {
  const int n = kPlaceBytes / rows / 16 * 16;   // 16 at least: 4096 rows
  return n < kCopyBytes ? n : kCopyBytes;
}

__global__ __launch_bounds__(256) void beam_place_kernel(const int32_t* source, BeamStates s) {
  extern __shared__ u32x4 lds[];
  const int width = column_bytes(s.rows);
  int64_t chunk = blockIdx.x;
  for (int i = 0; i < s.num_states; ++i) {
    if (s.from[i] != s.to[i]) continue;
    const int64_t bytes = s.row_bytes[i], chunks = (bytes + width - 1) / width;
    if (chunk >= chunks) {
      chunk -= chunks;
      continue;
    }
    const int64_t at = chunk * width;
    const int n = int(bytes - at < width ? bytes - at : width);
    const int align = alignment(reinterpret_cast<uintptr_t>(s.to[i]) | uint64_t(bytes));
    char* held = reinterpret_cast<char*>(lds);
    if (align == 16) permute_words<u32x4>(source, s.to[i], s.rows, bytes, at, n, held);
    else if (align == 4) permute_words<uint32_t>(source, s.to[i], s.rows, bytes, at, n, held);
    else permute_words<uint8_t>(source, s.to[i], s.rows, bytes, at, n, held);
    return;
  }
}

}  // namespace cocktail

using namespace cocktail;

namespace {

struct SelectPlan {
  int pieces;
  size_t sums, keys, tops, bytes;
};

int plan_select(int32_t groups, int32_t beams, int32_t vocab, int32_t keep, SelectPlan* s) {
  if (groups < 1 || beams < 1 || beams > 64 || int64_t(groups) * beams > (1 << 20))
    return fail(COCKTAIL_EINVAL, "%d groups of %d beams: beams must be in 1 .. 64, groups * beams in 1 .. 2^20", groups, beams);
  if (vocab < 1 || vocab > (1 << 24)) return fail(COCKTAIL_EINVAL, "vocab %d is not in 1 .. 2^24", vocab);
  if (keep < 1 || keep > kMostKeep) return fail(COCKTAIL_EINVAL, "keep %d is not in 1 .. %d", keep, kMostKeep);
  const int64_t rows = int64_t(groups) * beams;
  // Four workgroups to a compute unit, of 2048 logits (a tile of each wave) at least: 512 rows of 131072 in bf16 38 us, with half or twice as many workgroups
  // 44 and 43; 64 rows of 65001 11 us (11, 13); four rows of 32000 in fp32 6.3 us, with pieces of 4096 and 8192 logits 7.3 and 9.0.
  int64_t pieces = (1024 + rows - 1) / rows;
  const int64_t most = (int64_t(vocab) + 2047) / 2048;
  pieces = pieces < most ? pieces : most;
  s->pieces = int(pieces);
  s->sums = size_t(rows * pieces) * sizeof(double);
  s->keys = size_t(rows * pieces) * size_t(keep) * sizeof(LogitKey);
  s->tops = size_t(rows * pieces) * sizeof(float);
  s->bytes = s->sums + s->keys + s->tops + 16;
  return COCKTAIL_OK;
}

// Whether states are written over each other, or over what others are copied from while they are.  (What is in place may be copied from too: the
// copies are made first.)
bool states_overlap(const BeamStates& s) {
  enum { kRead, kWritten, kInPlace };
  struct Span {
    uint64_t first, end;
    int kind;
  } spans[2 * COCKTAIL_MAX_STATES];
  int n = 0;
  for (int i = 0; i < s.num_states; ++i) {
    const uint64_t from = reinterpret_cast<uintptr_t>(s.from[i]), to = reinterpret_cast<uintptr_t>(s.to[i]), bytes = uint64_t(s.row_bytes[i]) * s.rows;
    if (!bytes) continue;
    spans[n++] = {to, to + bytes, from == to ? kInPlace : kWritten};
    if (from != to) spans[n++] = {from, from + bytes, kRead};
  }
  std::sort(spans, spans + n, [](const Span& a, const Span& b) { return a.first < b.first; });
  uint64_t end[3] = {};   // of the spans of each kind so far
  for (int i = 0; i < n; ++i) {
    const Span& x = spans[i];
    if (x.first < end[kWritten] || (x.kind != kRead && x.first < end[kInPlace]) || (x.kind == kWritten && x.first < end[kRead])) return true;
    end[x.kind] = std::max(end[x.kind], x.end);
  }
  return false;
}

}  // namespace

extern "C" int cocktail_beam_select_workspace(int32_t groups, int32_t beams, int32_t vocab, int32_t keep, size_t* bytes) {
  if (!bytes) return fail(COCKTAIL_EINVAL, "bytes is NULL");
  SelectPlan s;
  if (int rc = plan_select(groups, beams, vocab, keep, &s)) return rc;
  *bytes = s.bytes;
  return COCKTAIL_OK;
}

extern "C" int cocktail_beam_select(const void* logits, int32_t dtype, int64_t stride_row, int32_t groups, int32_t beams, int32_t vocab,
                                    int32_t keep, const float* scores, const uint8_t* finished, int32_t eos, int32_t* source, int32_t* token,
                                    float* score, uint8_t* finished_out, void* workspace, size_t workspace_bytes, void* stream) {
  SelectPlan s;
  if (int rc = plan_select(groups, beams, vocab, keep, &s)) return rc;
  if (dtype != COCKTAIL_FP16 && dtype != COCKTAIL_BF16 && dtype != COCKTAIL_FP32)
    return fail(COCKTAIL_EINVAL, "dtype %d is none of COCKTAIL_FP16, COCKTAIL_BF16, COCKTAIL_FP32", dtype);
  if (!logits || !scores || !source || !token || !score) return fail(COCKTAIL_EINVAL, "logits, scores, source, token and score must not be NULL");
  if (stride_row < vocab || stride_row > (int64_t(1) << 40)) return fail(COCKTAIL_EINVAL, "stride_row %lld is not in vocab .. 2^40", (long long)stride_row);
  if (eos < -1 || eos >= vocab) return fail(COCKTAIL_EINVAL, "eos %d is not in -1 .. vocab - 1", eos);
  if (finished && eos < 0) return fail(COCKTAIL_EINVAL, "finished hypotheses need an eos");
  if (reinterpret_cast<uintptr_t>(logits) % (dtype == COCKTAIL_FP32 ? 4 : 2)) return fail(COCKTAIL_EALIGN, "logits must be aligned to their elements");
  if ((reinterpret_cast<uintptr_t>(scores) | reinterpret_cast<uintptr_t>(source) | reinterpret_cast<uintptr_t>(token) | reinterpret_cast<uintptr_t>(score)) & 3)
    return fail(COCKTAIL_EALIGN, "scores, source, token and score must be 4-byte aligned");
  if ((score == scores || (finished_out && finished_out == finished)) && keep != beams)
    return fail(COCKTAIL_EINVAL, "results can replace the scores only where keep == beams");
  if (!workspace) return fail(COCKTAIL_EINVAL, "workspace is NULL");
  if (reinterpret_cast<uintptr_t>(workspace) & 15) return fail(COCKTAIL_EALIGN, "workspace must be 16-byte aligned");
  if (workspace_bytes < s.bytes) return fail(COCKTAIL_ENOSPACE, "workspace has %zu bytes, %zu are needed", workspace_bytes, s.bytes);
  const int64_t rows = int64_t(groups) * beams, places = int64_t(groups) * keep;
  const int64_t all_logits = ((rows - 1) * stride_row + vocab) * (dtype == COCKTAIL_FP32 ? 4 : 2);
  // (a result in the place of its own input is none that overlaps with it)
  const MemoryRange written[] = {{source, 4 * places}, {token, 4 * places}, {score, 4 * places}, {finished_out, finished_out ? places : 0}, {workspace, int64_t(s.bytes)}};
  const MemoryRange read[] = {{logits, all_logits}, {scores, score == scores ? 0 : 4 * rows}, {finished, finished && finished_out != finished ? rows : 0}};
  if (overlap(written, read)) return fail(COCKTAIL_EINVAL, "results or workspace overlap with each other or with the inputs");
  BeamSelect a = {};
  a.logits = logits;
  a.stride_row = stride_row;
  a.groups = groups;
  a.beams = beams;
  a.vocab = vocab;
  a.keep = keep;
  a.pieces = s.pieces;
  a.scores = scores;
  a.finished = finished;
  a.eos = eos;
  a.source = source;
  a.token = token;
  a.score = score;
  a.finished_out = finished_out;
  char* w = static_cast<char*>(workspace);
  a.sums = reinterpret_cast<double*>(w);
  a.keys = reinterpret_cast<LogitKey*>(w + s.sums);
  a.tops = reinterpret_cast<float*>(w + s.sums + s.keys);
  hipStream_t st = static_cast<hipStream_t>(stream);
  const uint32_t blocks = uint32_t(groups) * uint32_t(beams) * uint32_t(s.pieces);
  hipError_t e = launch(dtype == COCKTAIL_FP32 ? beam_pieces_kernel<float> : dtype == COCKTAIL_BF16 ? beam_pieces_kernel<__bf16> : beam_pieces_kernel<_Float16>,
                        dim3(blocks), dim3(64 * kSelectWaves), st, a);
  if (e == hipSuccess) e = launch(beam_join_kernel, dim3(uint32_t(groups)), dim3(64 * kJoinWaves), st, a);
  if (e != hipSuccess) return fail(COCKTAIL_EHIP, "beam selection launch failed: %s", hipGetErrorString(e));
  return COCKTAIL_OK;
}

extern "C" int cocktail_beam_reorder(const int32_t* source, int32_t rows, const void* const* from, void* const* to, const int64_t* row_bytes,
                                     int32_t num_states, void* stream) {
  if (!source) return fail(COCKTAIL_EINVAL, "source is NULL");
  if (reinterpret_cast<uintptr_t>(source) & 3) return fail(COCKTAIL_EALIGN, "source must be 4-byte aligned");
  if (rows < 1 || rows > COCKTAIL_MAX_SEQS) return fail(COCKTAIL_EINVAL, "rows %d is not in 1 .. %d", rows, COCKTAIL_MAX_SEQS);
  if (num_states < 0 || num_states > COCKTAIL_MAX_STATES) return fail(COCKTAIL_EINVAL, "num_states %d is not in 0 .. %d", num_states, COCKTAIL_MAX_STATES);
  if (num_states && (!from || !to || !row_bytes)) return fail(COCKTAIL_EINVAL, "from, to and row_bytes must not be NULL");
  BeamStates s = {};
  s.num_states = num_states;
  s.rows = rows;
  int64_t copies = 0, columns = 0;
  const int width = column_bytes(rows);
  for (int i = 0; i < num_states; ++i) {
    if (row_bytes[i] < 0 || row_bytes[i] > (int64_t(1) << 40)) return fail(COCKTAIL_EINVAL, "row_bytes of state %d is not in 0 .. 2^40", i);
    if (row_bytes[i] && (!from[i] || !to[i])) return fail(COCKTAIL_EINVAL, "state %d is NULL", i);
    if (overlap(to[i], row_bytes[i] * rows, source, 4 * int64_t(rows))) return fail(COCKTAIL_EINVAL, "state %d overlaps with the sources", i);
    s.from[i] = static_cast<const char*>(from[i]);
    s.to[i] = static_cast<char*>(to[i]);
    s.row_bytes[i] = row_bytes[i];
    if (from[i] == to[i]) columns += (row_bytes[i] + width - 1) / width;
    else copies += (row_bytes[i] + kCopyBytes - 1) / kCopyBytes;
  }
  if (states_overlap(s)) return fail(COCKTAIL_EINVAL, "states are written over each other, or overlap with what they are copied from");
  if (copies * rows >= (int64_t(1) << 24) || copies >= (int64_t(1) << 24) || columns >= (int64_t(1) << 24))
    return fail(COCKTAIL_EINVAL, "the states are more than one launch takes");
  hipError_t e = hipSuccess;
  if (copies) e = launch(beam_copy_kernel, dim3(uint32_t(copies), uint32_t(rows)), dim3(256), static_cast<hipStream_t>(stream), source, s);
  if (e == hipSuccess && columns)
    e = launch_lds(beam_place_kernel, dim3(uint32_t(columns)), dim3(256), size_t(width) * rows, static_cast<hipStream_t>(stream), source, s);
  if (e != hipSuccess) return fail(COCKTAIL_EHIP, "beam reordering launch failed: %s", hipGetErrorString(e));
  return COCKTAIL_OK;
}
