// Decode kernel of cocktail_kv16_attention: up to 64 query rows (new tokens x query heads of a kv head) per (sequence, kv head).
//
// Bound by memory: a key costs 4 D bytes and 4 D * rows operations.  Measured: 128K tokens of 40 heads (2.68 GB) 388 us, eight sequences of 8 .. 130K, 8 kv heads,
// 4 query heads each (2.63 GB) 391 .. 397, 6.6 .. 6.9 TB/s; 64 of up to 4K, 8 kv heads, 8 query heads each (653 MB) 102 .. 104, 6.3 TB/s; 8 .. 48 rows behind 9 .. 16K
// (380 MB) 66 .. 68, 5.6 TB/s.
//  * Work is cut by tokens, not by sequences: the units of 32 tokens of all (sequence, kv head) segments lie one behind the other, and every wave
//    takes its share of that line, whatever the lengths are.  The numbering is made on the device from seq_lens, so that lengths can change
//    under a captured graph.  A segment inside one share is finished by its wave, the others leave a partial state per wave, or, where that would
//    make many of them, per workgroup whose waves all have parts of it.
//  * A lane's operands are whole pieces of memory.  Of K, lane (token c, quarter j) of sixteen tokens has channels 32 s + 8 j .. of its token, an operand of
//    S^T = K Q^T per s.  Of V, lane (c, j) has channels [8 c, 8 c + 8) of tokens 4 j .. 4 j + 3 (64 channels: [4 c, 4 c + 4)), whole rows per
//    load; pairs of tokens are put together by one byte permutation each, and are the operands of O^T = V^T P^T with the channels 8 c + t of product t.
//    The result layout of S^T (lane: a query row, tokens 4 j + x) is the operand layout of P^T with tokens numbered accordingly: weights
//    never leave their lane.
//  * The reference of the weights is only raised when a logit exceeds what it was made for by 2^4, so that the common step has no exchange
//    between lanes at all.  (What is there is multiplied by a power of two with a real exponent then, and weights are rounded against another reference: when
//    that takes place shows in the last bits, and is the same for the same inputs.)
#pragma once
#include <type_traits>

#include "kv16_attention.h"

namespace cocktail {

// A unit's keys are read by one wave whatever its rows are, and the memory is what is waited for.
struct Kv16Cost {
  static constexpr uint32_t kMost = 1;
  static constexpr bool kJoins = true;
  __device__ static int unit(const PagedAttention&, const PagedSeq&) { return 1; }
};

// Who takes what of the line:
//  kWaveShares: every wave a share of its own.
//  kGroupShares: every workgroup, whose waves share each part of a segment in it and join their states in LDS.  Where there are many rows and many keys: a
//    state of 64 rows is as large as 128 keys, and this way there are a quarter as many; but a second part in a share costs 6 us.
//  kWholeSegments: a workgroup has one segment, shared out in the same way: one launch, for short contexts.  (The states have to fit into LDS: eight waves
//    for up to 32 rows, else four.)
enum DecodeWork { kWaveShares, kGroupShares, kWholeSegments };
constexpr int whole_waves(int row_tiles) { return row_tiles <= 2 ? kWholeWaves : kDecodeWaves; }
template <int HD, bool BF16, int RT, DecodeWork WORK>
__global__ __launch_bounds__(64 * (WORK == kWholeSegments ? whole_waves(RT) : kDecodeWaves), RT == 1 ? 2 : 1) void kv16_decode_kernel(Kv16Attention args) {
  constexpr bool kWhole = WORK == kWholeSegments, kShared = WORK != kWaveShares;
  constexpr int kSteps = HD / 32;           // products per 16 tokens of S
  constexpr int kChannelTiles = HD / 16;
  constexpr int kWaves = kWhole ? whole_waves(RT) : kDecodeWaves;
  extern __shared__ int32_t pre[];
  __shared__ int32_t lds_words[kWholeWaves + 1];
  __shared__ float lds_state[kWaves][16 * RT][HD + 4];   // sums, then (m, l, l unrounded) of those that are joined here
  const PagedAttention& a = args.p;
  const PagedBatch& bt = a.batch;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c16 = lane & 15, j = lane >> 4;
  CostLine line = {};
  int w = 0;
  uint32_t u = 0, end = 1, share = 0;
  bool stream = false, joined = false;   // joined: the workgroup's waves have parts of one segment and leave one state
  if constexpr (!kWhole) {
    line = make_line<Kv16Cost>(a, pre, lds_words);
    share = cost_share<Kv16Cost>(line.total, a.workers);
    w = kShared ? blockIdx.x : __builtin_amdgcn_readfirstlane(blockIdx.x * kDecodeWaves + (threadIdx.x >> 6));
    u = w * share;
    end = u + share < line.total ? u + share : line.total;
    if (u >= end) return;
    // read once and not again before hundreds of MB have passed: past the caches
    stream = uint64_t(line.total) * (kUnit * 4 * HD) > kCachedBytes;
  }
  const int P = bt.page_size;
  const uint32_t run = uint32_t(P) * (2 * HD);
  const int64_t page_bytes = int64_t(run) * bt.num_kv_heads;
  const uint32_t off_k = c16 * (2 * HD) + j * 16, off_v = j * (8 * HD) + c16 * (HD / 8);

  bool first_segment = true;
  while (u < end) {
    CostPlace place;
    int h, p0, p1;   // the part of the segment
    if constexpr (kWhole) {
      const int number = blockIdx.x / bt.num_kv_heads;
      h = blockIdx.x - number * bt.num_kv_heads;
      // more sequences than rows: the workgroups are for those that have any
      place.b = bt.num_seqs > bt.total ? nth_active<kWaves>(a, number, lds_words) : number;
      if (place.b < 0) return;
      place.seq = of_lane(decode_seq(a, place.b), 0);
      if (place.seq.n == 0) return;
      const uint32_t units = decode_units(place.seq);
      place.cost = units;
      p0 = 0, p1 = units;
      u = end;
    } else {
      place = find_place(a, line, pre, u);
      const uint32_t units = place.cost, local = u - uint32_t(place.before) * uint32_t(bt.num_kv_heads);
      h = local / units;
      if (!kShared && a.joins) {
        const uint32_t begin = u - (local - uint32_t(h) * units);
        joined = workgroup_joins(begin, begin + units, blockIdx.x, share);
      }
      p0 = local - uint32_t(h) * units, p1 = end - u < units - p0 ? p0 + (end - u) : units;
      u += p1 - p0;
    }
    const int b = place.b, len = place.seq.len, rows = place.seq.n * a.rep;
    const uint32_t units = place.cost;
    const int u0 = kShared ? p0 + (p1 - p0) * wave / kWaves : p0, u1 = kShared ? p0 + (p1 - p0) * (wave + 1) / kWaves : p1;   // (what is a product fits: 2^26 units, 8 waves)

    // the queries: lane (row c16, quarter j) has the channels that its K pieces have
    u32x4 q[RT][kSteps] = {};
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int r = rt * 16 + c16, i = r / a.rep;
      if (r < rows) {
        const char* src = a.q + (place.seq.first + i) * a.stride_t + (h * a.rep + r - i * a.rep) * a.stride_h + j * 16;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) q[rt][s] = *reinterpret_cast<const u32x4*>(src + s * 64);
      }
    }

    // The tiles of the segment in order.  Every step loads two tiles and reads the table for two further on, whether they exist or not
    // (the last ones are then loaded again): with loads under a condition, the number of those in flight is not known when the code is made,
    // and every wait becomes one for all of them.
    const int32_t* table = bt.table + int64_t(b) * bt.table_stride;
    const int tiles = (len + 15) / 16;
    const int last_tile = u0 == u1 ? 0 : 2 * u1 < tiles ? 2 * u1 - 1 : tiles - 1;   // (a wave of those that share may have no keys: it reads the first)
    const int tiles_per_page = P / 16;
    int tile = u0 == u1 ? 0 : 2 * u0, col = tile / tiles_per_page, in_page = tile - col * tiles_per_page;   // of the table read
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
    const int64_t head = int64_t(h) * run;
    // Where the next two tiles lie (scalars), and whether their pages are any; a page that is none is read as the first one and left out.
    int64_t next0, next1;
    int next_ok0, next_ok1;
    int id0, id1, at0, at1;   // read a step ahead
    next_tile(id0, at0);
    next_tile(id1, at1);
    auto place_unit = [&]() __attribute__((always_inline)) {
      next_ok0 = uint32_t(id0) < uint32_t(bt.num_pages);
      next_ok1 = uint32_t(id1) < uint32_t(bt.num_pages);
      next0 = head + (next_ok0 ? id0 : 0) * page_bytes + at0 * (32 * HD);
      next1 = head + (next_ok1 ? id1 : 0) * page_bytes + at1 * (32 * HD);
      next_tile(id0, at0);
      next_tile(id1, at1);
    };
    u32x4 k0[kSteps], k1[kSteps], v0[4], v1[4];   // (HD 64: of V the first half)
    auto load = [&](auto policy, const char* from, uint32_t off) __attribute__((always_inline)) {
      const u32x4* src = reinterpret_cast<const u32x4*>(from + off);
      if constexpr (decltype(policy)::value) return __builtin_nontemporal_load(src);
      else return *src;
    };
    auto load_half = [&](auto policy, const char* from, uint32_t off) __attribute__((always_inline)) {
      const u32x2* src = reinterpret_cast<const u32x2*>(from + off);
      u32x2 x;
      if constexpr (decltype(policy)::value) x = __builtin_nontemporal_load(src);
      else x = *src;
      return u32x4{x[0], x[1], 0, 0};
    };
    auto load_k = [&](auto policy) __attribute__((always_inline)) {
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        k0[s] = load(policy, bt.pool + next0, off_k + s * 64);
        k1[s] = load(policy, bt.pool + next1, off_k + s * 64);
      }
    };
    auto load_v = [&](auto policy) __attribute__((always_inline)) {
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        if constexpr (HD == 128) {
          v0[x] = load(policy, args.v_pool + next0, off_v + x * (2 * HD));
          v1[x] = load(policy, args.v_pool + next1, off_v + x * (2 * HD));
        } else {
          v0[x] = load_half(policy, args.v_pool + next0, off_v + x * (2 * HD));
          v1[x] = load_half(policy, args.v_pool + next1, off_v + x * (2 * HD));
        }
      }
    };
    place_unit();
    if (stream) {
      load_k(std::integral_constant<bool, true>{});
      load_v(std::integral_constant<bool, true>{});
    } else {
      load_k(std::integral_constant<bool, false>{});
      load_v(std::integral_constant<bool, false>{});
    }

    const float c = fmaxf(a.scale, 1.2e-38f);
    float m[RT], lsum[RT];
    f32x4 l[RT], o[RT][kChannelTiles];
    int lim[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int r = rt * 16 + c16;
      lim[rt] = r < rows ? seen_by(place.seq, r / a.rep) : 0;
      m[rt] = kNoMax;
      lsum[rt] = 0.f;
      l[rt] = f32x4{};
#pragma unroll
      for (int ct = 0; ct < kChannelTiles; ++ct) o[rt][ct] = f32x4{};
    }
    const int free_below = seen_by(place.seq, 0);   // tokens that every query sees

    // A unit of keys: its logits, then K of the next one is sent for into the registers that they were made from, weights, and the same with V.
    auto step = [&](auto policy, int tok0) __attribute__((always_inline)) {
      const int ok0 = next_ok0, ok1 = next_ok1;
      place_unit();
      // logits
      f32x4 s[RT][2];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) s[rt][0] = s[rt][1] = f32x4{};
#pragma unroll
      for (int st = 0; st < kSteps; ++st)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          s[rt][0] = product16<BF16>(k0[st], q[rt][st], s[rt][0]);
          s[rt][1] = product16<BF16>(k1[st], q[rt][st], s[rt][1]);
        }
      __builtin_amdgcn_sched_barrier(0);
      load_k(policy);
      __builtin_amdgcn_sched_barrier(0);
      // keys that a query does not see, and what lies in places that no token has been stored to
      if (tok0 + kUnit > free_below || !ok0 || !ok1) {
        const int ka = tok0 + 4 * j, kb = ka + 16;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            s[rt][0][x] = ok0 && ka + x < lim[rt] ? s[rt][0][x] : -__builtin_inff();
            s[rt][1][x] = ok1 && kb + x < lim[rt] ? s[rt][1][x] : -__builtin_inff();
          }
          if (!(ok0 && ka + x < len)) v0[x] = u32x4{};
          if (!(ok1 && kb + x < len)) v1[x] = u32x4{};
        }
      }
      // weights
      u32x4 p[RT];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        float top = fmaxf(fmaxf(fmaxf(s[rt][0][0], s[rt][0][1]), fmaxf(s[rt][0][2], s[rt][0][3])),
                          fmaxf(fmaxf(s[rt][1][0], s[rt][1][1]), fmaxf(s[rt][1][2], s[rt][1][3]))) * c;
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
        for (int x = 0; x < 8; ++x) w8[x] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[rt][x >> 2][x & 3], c, -m[rt]));
        lsum[rt] += ((w8[0] + w8[1]) + (w8[2] + w8[3])) + ((w8[4] + w8[5]) + (w8[6] + w8[7]));
        p[rt] = u32x4{pack_weights<BF16>(w8[0], w8[1]), pack_weights<BF16>(w8[2], w8[3]), pack_weights<BF16>(w8[4], w8[5]), pack_weights<BF16>(w8[6], w8[7])};
        // the normaliser is the sum of the weights as they were rounded, so that a row whose values are all alike is that value
        l[rt] = product16<BF16>(ones16<BF16>(), p[rt], l[rt]);
      }
      // weighted sums
#pragma unroll
      for (int ct = 0; ct < kChannelTiles; ++ct) {
        const uint32_t pick = ct & 1 ? 0x07060302u : 0x05040100u;
        const int word = ct >> 1;
        const u32x4 vt = {__builtin_amdgcn_perm(v0[1][word], v0[0][word], pick), __builtin_amdgcn_perm(v0[3][word], v0[2][word], pick),
                          __builtin_amdgcn_perm(v1[1][word], v1[0][word], pick), __builtin_amdgcn_perm(v1[3][word], v1[2][word], pick)};
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) o[rt][ct] = product16<BF16>(vt, p[rt], o[rt][ct]);
      }
      __builtin_amdgcn_sched_barrier(0);
      load_v(policy);
      __builtin_amdgcn_sched_barrier(0);
    };

    if (stream) {
      for (int k = u0; k < u1; ++k) step(std::integral_constant<bool, true>{}, k * kUnit);
    } else {
      for (int k = u0; k < u1; ++k) step(std::integral_constant<bool, false>{}, k * kUnit);
    }

    // whole segments are finished here, others leave their state: a wave (or workgroup) has at most one that ends behind its share (or begins before
    // it) at each end, so two places are enough
    const bool whole = p0 == 0 && p1 == int(units);
    const int64_t slot = 2 * int64_t(w) + (first_segment ? 0 : 1);
    if (kShared || joined) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        float sum = lsum[rt];
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        float* dst = lds_state[wave][rt * 16 + c16];
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
          for (int y = 0; y < kChannelTiles / 4; ++y)
            *reinterpret_cast<f32x4*>(dst + j * (HD / 4) + x * kChannelTiles + 4 * y) = f32x4{o[rt][4 * y][x], o[rt][4 * y + 1][x], o[rt][4 * y + 2][x], o[rt][4 * y + 3][x]};
        if (j == 0) *reinterpret_cast<f32x4*>(dst + HD) = f32x4{m[rt], l[rt][0], sum, 0.f};
      }
      __syncthreads();
      // a wave joins a row or more at a time, a lane four channels
      constexpr int kLanes = HD / 4, kAtOnce = 64 / kLanes;
      const int at = lane % kLanes * 4;
      const int64_t first_state = (kShared ? slot : 2 * int64_t(w - wave)) * a.rows;
#pragma unroll kShared ? 2 : 1
      for (int r = wave * kAtOnce + lane / kLanes; r < rows; r += kWaves * kAtOnce) {
        f32x4 ml[kWaves], all = {}, sums = {};
        float top = kNoMax;
#pragma unroll
        for (int v = 0; v < kWaves; ++v) ml[v] = *reinterpret_cast<const f32x4*>(lds_state[v][r] + HD), top = fmaxf(top, ml[v][0]);
#pragma unroll
        for (int v = 0; v < kWaves; ++v) {
          const float weight = __builtin_amdgcn_exp2f(ml[v][0] - top);
          all += weight * *reinterpret_cast<const f32x4*>(lds_state[v][r] + at);
          sums += weight * ml[v];
        }
        if (kWhole || (kShared && whole)) {
          const int i = r / a.rep;
          const int64_t row = int64_t(place.seq.first + i) * bt.num_kv_heads * a.rep + h * a.rep + r - i * a.rep;
          const float inv = sums[1] == 0.f ? 0.f : 1.f / sums[1];
          *reinterpret_cast<u32x2*>(a.out + row * (2 * HD) + at * 2) = u32x2{pack_out(all[0] * inv, all[1] * inv, BF16), pack_out(all[2] * inv, all[3] * inv, BF16)};
          if (a.lse && at == 0) a.lse[row] = sums[1] == 0.f ? -__builtin_inff() : (top + __builtin_amdgcn_logf(sums[2])) * kLn2;
        } else {
          const int64_t state = first_state + r;
          *reinterpret_cast<f32x4*>(a.part_o + state * HD + at) = all;
          if (at == 0) {
            float* dst = a.part_ml + state * 3;
            dst[0] = top;
            dst[1] = sums[1];
            dst[2] = sums[2];
          }
        }
      }
      if constexpr (WORK != kGroupShares) return;
      __syncthreads();   // the next part's states take the place of these
      first_segment = false;
      continue;
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      float sum = lsum[rt];
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
      const int r = rt * 16 + c16;
      const float lr = l[rt][0];
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
            for (int y = 0; y < 4; ++y) v[y] = pack_out(o[rt][2 * y][x] * inv, o[rt][2 * y + 1][x] * inv, BF16);
            *reinterpret_cast<u32x4*>(dst + 16 * x) = v;
          } else {
            u32x2 v;
#pragma unroll
            for (int y = 0; y < 2; ++y) v[y] = pack_out(o[rt][2 * y][x] * inv, o[rt][2 * y + 1][x] * inv, BF16);
            *reinterpret_cast<u32x2*>(dst + 8 * x) = v;
          }
        }
        if (a.lse && j == 0) a.lse[row] = lr == 0.f ? -__builtin_inff() : (m[rt] + __builtin_amdgcn_logf(sum)) * kLn2;
      } else {
        // through LDS, so that a store is a kilobyte of whole rows
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
