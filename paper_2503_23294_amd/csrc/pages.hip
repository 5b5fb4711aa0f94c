// cocktail_pages_*: which pages the sequences of a batch have, on the device.  The tables are small (a few hundred KB) and every call is a
// matter of launches and of the latency of a few dependent passes, but for the pages it copies, which are bound by memory.
#include <hip/hip_runtime.h>

#include "fp4_common.h"

namespace cocktail {

// Workspace: [0] number of pages to move, then the moves (from, to), then a list of pages / the new number of every page.
struct PageWork {
  int32_t* count;
  int32_t* moves;   // pairs
  int32_t* list;    // num_pages
};
__host__ __device__ inline size_t page_work_ints(int num_seqs, int num_pages) {
  const size_t moves = size_t(num_seqs > num_pages ? num_seqs : num_pages);
  return 16 + 2 * moves + size_t(num_pages);
}
inline PageWork page_work(void* workspace, int num_seqs, int num_pages) {
  int32_t* w = static_cast<int32_t*>(workspace);
  return {w, w + 16, w + 16 + 2 * size_t(num_seqs > num_pages ? num_seqs : num_pages)};
}

// Exclusive prefix of v over the threads of the workgroup, and the sum; every thread gets both.  `lds`: THREADS / 64 ints, not the same in two
// calls one behind the other (so that one barrier is enough).
template <int THREADS>
__device__ __forceinline__ int block_prefix(int v, int* sum, int* lds) {
  constexpr int kWaves = THREADS / 64;
  const int wave = threadIdx.x >> 6;
  const int x = wave_prefix(v);
  if ((threadIdx.x & 63) == 63) lds[wave] = x;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const int n = lds[w];
    before += w < wave ? n : 0;
    all += n;
  }
  *sum = all;
  return before + x - v;
}

// References of 16 consecutive pages, a word each; pages behind the last one count as held.
struct Refs16 {
  int r[16];
};
__device__ __forceinline__ Refs16 load_refs(const cocktail_page_table& p, int64_t page) {
  Refs16 x;
#pragma unroll
  for (int i = 0; i < 16; ++i) x.r[i] = page + i < p.num_pages ? p.refs[page + i] : 1;
  return x;
}

// One workgroup, for it is a matter of a few dependent reads: lengths, last pages, their holders, free pages.  Thread t has rows t * ROWS + i, so that
// prefixes over the rows are prefixes over the threads.  A step of 64 sequences: 8 us with 256 threads, lists in shared memory and the
// references read before anything is known; 18 us with 1024 threads that read everything again where it is needed.
constexpr int kListInLds = 2048;
template <int THREADS, int ROWS>
__global__ __launch_bounds__(THREADS) void pages_resize_kernel(cocktail_page_table p, const int32_t* __restrict__ delta, PageWork w, int copy) {
  constexpr int kMost = THREADS * ROWS;
  __shared__ int32_t tail_of[kMost], first[kMost], start_of[kMost], lds_list[kListInLds], scratch[4][THREADS / 64];
  __shared__ int any_shared, failed;   // failed: 1 columns, 2 pools
  const int tid = threadIdx.x;
  Refs16 refs = load_refs(p, int64_t(tid) * 16);
  if (tid == 0) any_shared = failed = 0;
  int64_t len1[ROWS];
  int have[ROWS], need[ROWS], tail[ROWS], held[ROWS];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const int b = tid * ROWS + i;
    have[i] = need[i] = held[i] = 0;
    len1[i] = 0;
    tail[i] = -1;
    if (b >= p.num_seqs) continue;
    const int d = delta[b];
    const int len0 = max(p.seq_lens[b], 0);
    len1[i] = max(int64_t(len0) + d, int64_t(0));
    have[i] = min(int((int64_t(len0) + p.page_size - 1) / p.page_size), p.table_stride);
    const int64_t want = (len1[i] + p.page_size - 1) / p.page_size;
    need[i] = want > p.table_stride ? -1 : int(want);
    if (d > 0 && len0 % p.page_size && have[i] > 0) tail[i] = p.table[int64_t(b) * p.table_stride + have[i] - 1];
    if (uint32_t(tail[i]) >= uint32_t(p.num_pages)) tail[i] = -1;
  }
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const int b = tid * ROWS + i;
    if (tail[i] >= 0) held[i] = p.refs[tail[i]];
    tail_of[b] = tail[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    if (held[i] > 1) any_shared = 1;   // (every thread that writes these writes the same)
    if (need[i] < 0) failed = 1;
  }
  __syncthreads();
  if (any_shared && !copy) failed = 2;
  bool copies[ROWS];
  int fresh[ROWS], fresh_sum = 0, ncopies = 0;
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const int b = tid * ROWS + i;
    copies[i] = false;
    if (held[i] > 1) {
      int alike = 0;
      bool later = false;
#pragma unroll 8
      for (int c = 0; c < p.num_seqs; ++c) {
        const bool same = tail_of[c] == tail[i];
        alike += same ? 1 : 0;
        later |= same && c > b;
      }
      copies[i] = later || held[i] > alike;
    }
    fresh[i] = (copies[i] ? 1 : 0) + max(need[i] - have[i], 0);
    fresh_sum += fresh[i];
    ncopies += copies[i] ? 1 : 0;
  }
  int total, nmoves;
  int at = block_prefix<THREADS>(fresh_sum, &total, scratch[0]);
  int move = block_prefix<THREADS>(ncopies, &nmoves, scratch[1]);
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    first[tid * ROWS + i] = at;
    start_of[tid * ROWS + i] = have[i] - (copies[i] ? 1 : 0);   // column of the first page that it takes: a copy replaces the last one
    at += fresh[i];
  }
  // the lowest free pages, as many as are needed; the next references are on their way while some are counted
  const bool in_lds = total <= kListInLds;
  int found = 0;
  if (!failed && total)
    for (int64_t base = 0, turn = 0;; ++turn) {
      const int64_t page = base + int64_t(tid) * 16;
      int mine = 0, sum;
      const Refs16 now = refs;
#pragma unroll
      for (int i = 0; i < 16; ++i) mine += now.r[i] == 0 ? 1 : 0;
      base += THREADS * 16;
      const bool more = base < p.num_pages;
      if (more) refs = load_refs(p, base + int64_t(tid) * 16);
      int k = found + block_prefix<THREADS>(mine, &sum, scratch[2 + (turn & 1)]);
      if (mine)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (now.r[i] == 0) {
            if (k < total) {
              if (in_lds) lds_list[k] = int(page) + i;
              else w.list[k] = int(page) + i;
            }
            ++k;
          }
      found += sum;
      if (found >= total || !more) break;
    }
  __syncthreads();   // the list and first[] are there
  if (failed || found < total) {
    if (tid == 0) {
      p.status[0] = failed ? -failed : total - found;
      w.count[0] = 0;
    }
    return;
  }
  // fresh pages: thread by thread over all of them, since one sequence may take thousands
  for (int k = tid; k < total; k += THREADS) {
    int b = 0, e = kMost;
    while (e - b > 1) {
      const int m = (b + e) >> 1;
      if (first[m] <= k) b = m;
      else e = m;
    }
    // (rows before b that take nothing have the same first[]; the search ends at the last of them, which is the one that does)
    const int page = in_lds ? lds_list[k] : w.list[k];
    p.refs[page] = 1;
    p.table[int64_t(b) * p.table_stride + start_of[b] + (k - first[b])] = page;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const int b = tid * ROWS + i;
    if (b >= p.num_seqs) continue;
    p.seq_lens[b] = int(len1[i]);
    if (copies[i]) {
      w.moves[2 * move] = tail[i];
      w.moves[2 * move + 1] = in_lds ? lds_list[first[b]] : w.list[first[b]];
      ++move;
      atomicAdd(&p.refs[tail[i]], -1);
    }
  }
  if (tid == 0) {
    w.count[0] = nmoves;
    p.status[0] = 0;
  }
  // pages that are given back: a wave per row
  __syncthreads();
#pragma unroll
  for (int i = 0; i < ROWS; ++i) tail_of[tid * ROWS + i] = max(need[i], 0);
  __syncthreads();
  for (int b = tid >> 6; b < p.num_seqs; b += THREADS / 64)
    for (int c = tail_of[b] + (tid & 63); c < start_of[b]; c += 64) {
      int32_t* entry = p.table + int64_t(b) * p.table_stride + c;
      const int page = *entry;
      if (uint32_t(page) < uint32_t(p.num_pages)) atomicAdd(&p.refs[page], -1);
      *entry = -1;
    }
}

// A workgroup has a few columns of the table, for all rows: it reads them all before it writes any, so that rows can change places.
// No two workgroups touch the same entry, and references are sums, in any order the same.  64 sequences: 5 us.
__global__ __launch_bounds__(256) void pages_fork_kernel(cocktail_page_table p, const int32_t* __restrict__ source, int cols) {
  extern __shared__ int32_t lds[];   // [num_seqs][cols], by the first workgroup first for the lengths
  const int n = p.num_seqs;
  if (blockIdx.x == 0) {
    for (int b = threadIdx.x; b < n; b += 256) lds[b] = p.seq_lens[b];
    __syncthreads();
    for (int b = threadIdx.x; b < n; b += 256) {
      const int s = source[b];
      if (s != b && s < n) p.seq_lens[b] = s < 0 ? 0 : lds[s];
    }
    __syncthreads();
  }
  const int64_t c0 = int64_t(blockIdx.x) * cols;
  for (int i = threadIdx.x; i < n * cols; i += 256) {
    const int b = i / cols, c = i % cols;
    lds[i] = c0 + c < p.table_stride ? p.table[int64_t(b) * p.table_stride + c0 + c] : -1;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n * cols; i += 256) {
    const int b = i / cols, c = i % cols;
    const int s = source[b];
    if (s == b || s >= n || c0 + c >= p.table_stride) continue;
    const int was = lds[i], is = s < 0 ? -1 : lds[s * cols + c];
    if (was == is) continue;
    p.table[int64_t(b) * p.table_stride + c0 + c] = is;
    if (uint32_t(was) < uint32_t(p.num_pages)) atomicAdd(&p.refs[was], -1);
    if (uint32_t(is) < uint32_t(p.num_pages)) atomicAdd(&p.refs[is], 1);
  }
}

// One workgroup: where every page in use goes.
constexpr int kCompactThreads = 1024;
__global__ __launch_bounds__(kCompactThreads) void pages_compact_kernel(cocktail_page_table p, PageWork w) {
  __shared__ int scratch[4][kCompactThreads / 64];
  const int tid = threadIdx.x;
  int mine = 0, used;
  for (int64_t page = int64_t(tid) * 16; page < p.num_pages; page += kCompactThreads * 16) {
    const Refs16 x = load_refs(p, page);
#pragma unroll
    for (int i = 0; i < 16; ++i) mine += x.r[i] != 0 && page + i < p.num_pages ? 1 : 0;
  }
  block_prefix<kCompactThreads>(mine, &used, scratch[0]);
  int holes = 0, movers = 0;
  for (int64_t base = 0, turn = 0; base < p.num_pages; base += kCompactThreads * 4, ++turn) {
    int kind[4], h = 0, m = 0, sum;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t page = base + tid * 4 + i;
      kind[i] = 0;
      if (page < p.num_pages) {
        const bool in_use = p.refs[page] != 0;
        if (page < used && !in_use) kind[i] = 1, ++h;
        if (page >= used && in_use) kind[i] = 2, ++m;
        w.list[page] = int(page);
      }
    }
    // both numbers in one word: at most 2^12 of each in a turn
    const int before = block_prefix<kCompactThreads>(h | m << 16, &sum, scratch[2 + (turn & 1)]);
    int hk = holes + (before & 0xffff), mk = movers + (before >> 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (kind[i] == 1) w.moves[2 * hk++ + 1] = int(base) + tid * 4 + i;
      if (kind[i] == 2) w.moves[2 * mk++] = int(base) + tid * 4 + i;
    }
    holes += sum & 0xffff;
    movers += sum >> 16;
  }
  __syncthreads();
  for (int k = tid; k < movers; k += kCompactThreads) w.list[w.moves[2 * k]] = w.moves[2 * k + 1];
  if (tid == 0) w.count[0] = movers;
}

struct Pools {
  char* p[COCKTAIL_MAX_POOLS];
};

// Copies the moves' pages in all pools, a piece of up to 16 KB at a time; after a compaction (remap) the table and the references follow.
// The grid strides over the pieces; their number is on the device.  Bound by memory: 226 MB moved in 76 us (6.0 TB/s read and written).
__global__ __launch_bounds__(256) void pages_move_kernel(Pools pools, int num_pools, int64_t page_bytes, const int32_t* __restrict__ count,
                                                         const int32_t* __restrict__ moves, const int32_t* __restrict__ remap, cocktail_page_table p) {
  const int n = count[0];
  if (remap) {
    const int64_t entries = int64_t(p.num_seqs) * p.table_stride;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < entries; i += int64_t(gridDim.x) * 256) {
      const int page = p.table[i];
      if (uint32_t(page) < uint32_t(p.num_pages)) {
        const int to = remap[page];
        if (to != page) p.table[i] = to;
      }
    }
    for (int i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256) {
      const int from = moves[2 * i], to = moves[2 * i + 1];
      p.refs[to] = p.refs[from];
      p.refs[from] = 0;
    }
  }
  constexpr int kPiece = 16384;
  const int pieces = int((page_bytes + kPiece - 1) / kPiece);
  const int64_t items = int64_t(n) * num_pools * pieces;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int piece = int(it % pieces);
    const int64_t rest = it / pieces;
    const int pool = int(rest % num_pools), m = int(rest / num_pools);
    char* base = pools.p[pool] + int64_t(piece) * kPiece;
    const u32x4* src = reinterpret_cast<const u32x4*>(base + moves[2 * m] * page_bytes);
    u32x4* dst = reinterpret_cast<u32x4*>(base + moves[2 * m + 1] * page_bytes);
    const int64_t left = page_bytes - int64_t(piece) * kPiece;
    const int words = int((left < kPiece ? left : kPiece) / 16);
    // read past the caches (104 -> 85 us for 226 MB; written past them as well 98)
#pragma unroll 4
    for (int i = threadIdx.x; i < words; i += 256) dst[i] = __builtin_nontemporal_load(src + i);
  }
}

int check_page_table(const cocktail_page_table* p) {
  if (!p) return fail(COCKTAIL_EINVAL, "page table is NULL");
  if (!p->table || !p->seq_lens || !p->refs || !p->status) return fail(COCKTAIL_EINVAL, "table, seq_lens, refs and status must not be NULL");
  if (p->num_seqs < 1 || p->num_seqs > COCKTAIL_MAX_SEQS) return fail(COCKTAIL_EINVAL, "num_seqs %d is not in 1 .. %d", p->num_seqs, COCKTAIL_MAX_SEQS);
  if (p->table_stride < 1 || p->page_size < 1 || p->num_pages < 1 || p->num_pages > (1 << 30))
    return fail(COCKTAIL_EINVAL, "table_stride, page_size and num_pages must be positive (pages up to 2^30)");
  if (int64_t(p->table_stride) * p->page_size >= (int64_t(1) << 31))
    return fail(COCKTAIL_EINVAL, "table_stride * page_size = %lld tokens: must be below 2^31", (long long)(int64_t(p->table_stride) * p->page_size));
  // (a resize adds up in 32 bits how many pages all sequences take)
  if (int64_t(p->num_seqs) * p->table_stride >= (int64_t(1) << 31))
    return fail(COCKTAIL_EINVAL, "num_seqs * table_stride = %lld entries: must be below 2^31", (long long)(int64_t(p->num_seqs) * p->table_stride));
  if ((reinterpret_cast<uintptr_t>(p->table) | reinterpret_cast<uintptr_t>(p->seq_lens) | reinterpret_cast<uintptr_t>(p->refs) |
       reinterpret_cast<uintptr_t>(p->status)) & 3)
    return fail(COCKTAIL_EALIGN, "table, seq_lens, refs and status must be 4-byte aligned");
  return COCKTAIL_OK;
}

}  // namespace cocktail

using namespace cocktail;

namespace {

int check_pools(const cocktail_page_table* p, void* const* pools, int32_t num_pools, int64_t page_bytes, const void* workspace,
                size_t workspace_bytes, Pools* out) {
  if (int rc = check_page_table(p)) return rc;
  if (num_pools < 0 || num_pools > COCKTAIL_MAX_POOLS) return fail(COCKTAIL_EINVAL, "num_pools %d is not in 0 .. %d", num_pools, COCKTAIL_MAX_POOLS);
  if (num_pools && !pools) return fail(COCKTAIL_EINVAL, "pools is NULL");
  if (num_pools && (page_bytes < 16 || page_bytes % 16 || page_bytes > (int64_t(1) << 32)))
    return fail(COCKTAIL_EINVAL, "page_bytes %lld is not a positive multiple of 16 up to 2^32", (long long)page_bytes);
  for (int i = 0; i < num_pools; ++i) {
    if (!pools[i]) return fail(COCKTAIL_EINVAL, "pool %d is NULL", i);
    if (reinterpret_cast<uintptr_t>(pools[i]) & 15) return fail(COCKTAIL_EALIGN, "pool %d is not 16-byte aligned", i);
    out->p[i] = static_cast<char*>(pools[i]);
  }
  if (!workspace) return fail(COCKTAIL_EINVAL, "workspace is NULL");
  if (reinterpret_cast<uintptr_t>(workspace) & 15) return fail(COCKTAIL_EALIGN, "workspace must be 16-byte aligned");
  const size_t need = 4 * page_work_ints(p->num_seqs, p->num_pages);
  if (workspace_bytes < need) return fail(COCKTAIL_ENOSPACE, "workspace has %zu bytes, %zu are needed", workspace_bytes, need);
  return COCKTAIL_OK;
}

}  // namespace

extern "C" int cocktail_pages_workspace(const cocktail_page_table* pages, size_t* bytes) {
  if (!bytes) return fail(COCKTAIL_EINVAL, "bytes is NULL");
  if (int rc = check_page_table(pages)) return rc;
  *bytes = 4 * page_work_ints(pages->num_seqs, pages->num_pages);
  return COCKTAIL_OK;
}

extern "C" int cocktail_pages_resize(const cocktail_page_table* pages, const int32_t* delta, void* const* pools, int32_t num_pools,
                                     int64_t page_bytes, void* workspace, size_t workspace_bytes, void* stream) {
  Pools list = {};
  if (int rc = check_pools(pages, pools, num_pools, page_bytes, workspace, workspace_bytes, &list)) return rc;
  if (!delta) return fail(COCKTAIL_EINVAL, "delta is NULL");
  if (reinterpret_cast<uintptr_t>(delta) & 3) return fail(COCKTAIL_EALIGN, "delta must be 4-byte aligned");
  hipStream_t st = static_cast<hipStream_t>(stream);
  const PageWork w = page_work(workspace, pages->num_seqs, pages->num_pages);
  // few rows and few pages: fewer threads wait for each other
  hipError_t e = pages->num_seqs <= 256 && pages->num_pages <= 16384
                     ? launch(pages_resize_kernel<256, 1>, dim3(1), dim3(256), st, *pages, delta, w, int(num_pools > 0))
                     : launch(pages_resize_kernel<1024, COCKTAIL_MAX_SEQS / 1024>, dim3(1), dim3(1024), st, *pages, delta, w, int(num_pools > 0));
  if (e == hipSuccess && num_pools) {
    const int64_t items = int64_t(pages->num_seqs) * num_pools * ((page_bytes + 16383) / 16384);
    e = launch(pages_move_kernel, dim3(uint32_t(items < 2048 ? items : 2048)), dim3(256), st, list, num_pools, page_bytes, w.count, w.moves, nullptr, *pages);
  }
  if (e != hipSuccess) return fail(COCKTAIL_EHIP, "resize launch failed: %s", hipGetErrorString(e));
  return COCKTAIL_OK;
}

extern "C" int cocktail_pages_fork(const cocktail_page_table* pages, const int32_t* source, void* stream) {
  if (int rc = check_page_table(pages)) return rc;
  if (!source) return fail(COCKTAIL_EINVAL, "source is NULL");
  if (reinterpret_cast<uintptr_t>(source) & 3) return fail(COCKTAIL_EALIGN, "source must be 4-byte aligned");
  // 64 KB of LDS at most: 16 columns (64 bytes of a row) up to 1024 sequences
  int cols = 16;
  while (cols > 1 && pages->num_seqs * cols > 16384) cols >>= 1;
  const uint32_t blocks = (pages->table_stride + cols - 1) / cols;
  const hipError_t e = launch_lds(pages_fork_kernel, dim3(blocks), dim3(256), sizeof(int32_t) * pages->num_seqs * cols, static_cast<hipStream_t>(stream),
                                  *pages, source, cols);
  if (e != hipSuccess) return fail(COCKTAIL_EHIP, "fork launch failed: %s", hipGetErrorString(e));
  return COCKTAIL_OK;
}

extern "C" int cocktail_pages_compact(const cocktail_page_table* pages, void* const* pools, int32_t num_pools, int64_t page_bytes,
                                      void* workspace, size_t workspace_bytes, void* stream) {
  Pools list = {};
  if (int rc = check_pools(pages, pools, num_pools, page_bytes, workspace, workspace_bytes, &list)) return rc;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const PageWork w = page_work(workspace, pages->num_seqs, pages->num_pages);
  hipError_t e = launch(pages_compact_kernel, dim3(1), dim3(kCompactThreads), st, *pages, w);
  if (e == hipSuccess)
    e = launch(pages_move_kernel, dim3(2048), dim3(256), st, list, num_pools, page_bytes, w.count, w.moves, w.list, *pages);
  if (e != hipSuccess) return fail(COCKTAIL_EHIP, "compact launch failed: %s", hipGetErrorString(e));
  return COCKTAIL_OK;
}

extern "C" int cocktail_pages_check(const cocktail_page_table* pages, void* stream) {
  if (int rc = check_page_table(pages)) return rc;
  hipStream_t st = static_cast<hipStream_t>(stream);
  int32_t word = 0;
  hipError_t e = hipMemcpyAsync(&word, pages->status, sizeof(word), hipMemcpyDeviceToHost, st);
  if (e == hipSuccess) e = hipStreamSynchronize(st);
  if (e != hipSuccess) {
    (void)hipGetLastError();
    return fail(COCKTAIL_EHIP, "reading the status failed: %s", hipGetErrorString(e));
  }
  if (word == -2) return fail(COCKTAIL_ESTATE, "the last resize did nothing: a shared page had to be copied and no pools were given");
  if (word < 0) return fail(COCKTAIL_ESTATE, "the last resize did nothing: the page table has too few columns for a sequence");
  if (word) return fail(COCKTAIL_ESTATE, "the last resize did nothing: %d pages were missing", word);
  return COCKTAIL_OK;
}
