// The pages of a key/value cache: growing, forking, trimming and compacting rows, copying pages.  Whole numbers
// throughout, and no result depends on the order of blocks: pages are taken lowest number first by prefix sums,
// counts change by integer atomics.  Bound by latency: chains of dependent loads and scans, 3 to 8 us a launch.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/maaso_instance.h"
#include "element_types.hpp"
#include "lds_barrier.hpp"

namespace maaso {

constexpr uint32_t kPageThreads = 1024;

struct PageArgs {
  uint32_t n_pages, page_log2, n_rows, width;
  int32_t* refs;
  int32_t* table;
  int32_t* length;
  uint32_t* status;
};

__device__ inline void raise(uint32_t* status, uint32_t bit) { atomicOr(status, bit); }

// Exclusive prefix sum over the block's threads (a multiple of 64, at most 1024); `total` receives the sum.
__device__ inline uint32_t block_scan(uint32_t v, uint32_t* part /*[17] LDS*/, uint32_t& total) {
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  uint32_t x = v;
  for (uint32_t d = 1; d < 64u; d <<= 1) {
    const uint32_t y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  __syncthreads();  // (the sums of an earlier call are read)
  if (lane == 63u) part[wave] = x;
  __syncthreads();
  uint32_t before = 0, sum = 0;
  for (uint32_t w = 0; w < waves; ++w) {
    if (w == wave) before = sum;
    sum += part[w];
  }
  total = sum;
  return before + x - v;
}

// ------------------------------------------------------------------------------------------------ extend
struct ExtendArgs {
  PageArgs p;
  const int32_t* rows;
  const int32_t* q_start;
  uint32_t n, n_tok;
  int64_t* slot;
  int32_t* pos;
  int32_t* copies;
  // workspace
  uint32_t* ok;     // [1]
  int32_t* held;    // [n] tokens before the call
  uint32_t* begin;  // [n + 1] index of the row's first page among those taken
  int32_t* first;   // [n] index in the row of its first new page
  int32_t* ids;     // [n_pages] the pages taken
};

// Whether every row can grow, which pages are taken, and from where each row has them.  One block: the prefix
// sums over rows and over the pool are a chain, and a step's rows are few (64 rows of a pool of 8192 pages: 7.8 us in
// extend_kernel; 48 prompts' 1500 pages of 65,536: 5.8 to plan, 4.7 to write).
__device__ inline bool extend_plan(const ExtendArgs& a, uint32_t* part, uint32_t* bad) {
  const uint32_t t = threadIdx.x, per = 1u << a.p.page_log2;
  // (which of four pages are free; the first step's are asked for before the rows are looked at)
  auto free_of = [&](uint32_t p0) {
    uint32_t free4 = 0;
#pragma unroll
    for (uint32_t k = 0; k < 4u; ++k)
      if (p0 + k < a.p.n_pages && a.p.refs[p0 + k] == 0) free4 |= 1u << k;
    return free4;
  };
  uint32_t free4 = free_of(t * 4u);
  if (t == 0) *bad = 0u;
  __syncthreads();
  uint32_t need_all = 0;
  for (uint32_t base = 0; base < a.n; base += blockDim.x) {
    const uint32_t i = base + t;
    uint32_t need = 0;
    if (i < a.n) {
      const int32_t row = a.rows[i], q0 = a.q_start[i], q1 = a.q_start[i + 1];
      uint32_t wrong = 0;
      if (q0 < 0 || q1 < q0 || (uint32_t)q1 > a.n_tok || (i == 0u && q0 != 0) || (i + 1u == a.n && (uint32_t)q1 != a.n_tok))
        wrong = MAASO_INST_BAD_BOUND;
      if (row < 0 || (uint32_t)row >= a.p.n_rows) wrong |= MAASO_INST_BAD_ROW;
      if (!wrong) {
        const int64_t held = a.p.length[row], end = held + (q1 - q0);
        const int64_t had = (held + per - 1) >> a.p.page_log2, has = (end + per - 1) >> a.p.page_log2;
        if (held < 0 || had > a.p.width) wrong = MAASO_INST_BAD_ROW;
        else if (has > a.p.width) wrong = MAASO_INST_NO_PAGES;
        else {
          int32_t from = -1;
          if ((held & (per - 1u)) && q1 > q0) {
            const int32_t last = a.p.table[(size_t)row * a.p.width + (had - 1)];
            if (last < 0 || (uint32_t)last >= a.p.n_pages) wrong = MAASO_INST_BAD_PAGE;
            else if (a.p.refs[last] > 1) from = last;
          }
          need = (uint32_t)(has - had) + (from >= 0 ? 1u : 0u);
          a.held[i] = (int32_t)held;
          a.first[i] = (int32_t)had - (from >= 0 ? 1 : 0);
          a.copies[2 * i] = from;
        }
      }
      if (wrong) {
        atomicOr(bad, wrong);
        need = 0;
      }
    }
    uint32_t sum;
    const uint32_t before = block_scan(need, part, sum);
    if (i < a.n) a.begin[i] = need_all + before;
    need_all += sum;  // (at most n * width pages: the host keeps that below 2^31)
  }
  if (t == 0) a.begin[a.n] = need_all;
  // The first need_all free pages, 4 per thread and step.
  uint32_t found = 0;
  for (uint32_t base = 0; base < a.p.n_pages && found < need_all; base += blockDim.x * 4u) {
    const uint32_t p0 = base + t * 4u, now = free4;
    free4 = free_of(p0 + blockDim.x * 4u);  // (the next step's, while this one's are summed; pages are below 2^24)
    uint32_t sum;
    uint32_t at = found + block_scan(__popc(now), part, sum);
    for (uint32_t k = 0; k < 4u; ++k)
      if (now >> k & 1u) {
        if (at < need_all) a.ids[at] = (int32_t)(p0 + k);
        ++at;
      }
    found += sum;
  }
  if (t == 0 && found < need_all) atomicOr(bad, MAASO_INST_NO_PAGES);
  lds_atomics_barrier();
  if (t == 0 && *bad) raise(a.p.status, *bad);
  return *bad == 0u;
}

// Row i's new page entries, counts and length, by all threads of `threads`, of which this is `t`.
__device__ inline void extend_apply(const ExtendArgs& a, bool ok, uint32_t t, uint32_t threads) {
  const uint32_t per = 1u << a.p.page_log2;
  for (uint32_t i = t; i < a.n; i += threads) {
    int32_t from = -1, to = -1;
    if (ok) {
      from = a.copies[2 * i];
      if (from >= 0) {
        to = a.ids[a.begin[i]];
        atomicSub(&a.p.refs[from], 1);
      }
      a.p.length[a.rows[i]] = a.held[i] + (a.q_start[i + 1] - a.q_start[i]);
    }
    a.copies[2 * i] = from;
    a.copies[2 * i + 1] = to;
  }
  if (ok) {
    const uint32_t taken = a.begin[a.n];
    for (uint32_t j = t; j < taken; j += threads) {
      uint32_t lo = 0, hi = a.n;  // the row: the last one that begins at j or before
      while (hi - lo > 1u) {
        const uint32_t mid = (lo + hi) >> 1;
        if (a.begin[mid] <= j) lo = mid; else hi = mid;
      }
      const int32_t id = a.ids[j];
      a.p.table[(size_t)a.rows[lo] * a.p.width + (uint32_t)a.first[lo] + (j - a.begin[lo])] = id;
      a.p.refs[id] = 1;
    }
  }
  for (uint32_t k = t; k < a.n_tok; k += threads) {
    int64_t slot = -1;
    int32_t pos = -1;
    if (ok) {
      uint32_t lo = 0, hi = a.n;  // the row: the last one whose tokens begin at k or before
      while (hi - lo > 1u) {
        const uint32_t mid = (lo + hi) >> 1;
        if ((uint32_t)a.q_start[mid] <= k) lo = mid; else hi = mid;
      }
      pos = a.held[lo] + (int32_t)(k - (uint32_t)a.q_start[lo]);
      const int32_t nth = pos >> a.p.page_log2;
      // (a new page's entry is read from the list: the table's may not be written yet)
      const int32_t page = nth >= a.first[lo] ? a.ids[a.begin[lo] + (uint32_t)(nth - a.first[lo])]
                                              : a.p.table[(size_t)a.rows[lo] * a.p.width + (uint32_t)nth];
      slot = (int64_t)page * per + (pos & (int32_t)(per - 1u));
    }
    a.slot[k] = slot;
    if (a.pos) a.pos[k] = pos;
  }
}

// Few tokens: all in one block, one launch.  The searches for a page's and a token's row are chains of reads, so what they
// read lies in shared memory where the rows are no more than the threads.
__global__ void __launch_bounds__(kPageThreads) extend_kernel(ExtendArgs a) {
  __shared__ uint32_t part[17], bad;
  __shared__ uint32_t begin[kPageThreads + 1];
  __shared__ int32_t held[kPageThreads], first[kPageThreads], start[kPageThreads + 1];
  if (a.n <= kPageThreads) {
    for (uint32_t i = threadIdx.x; i <= a.n; i += kPageThreads) start[i] = a.q_start[i];
    a.begin = begin;
    a.held = held;
    a.first = first;
    a.q_start = start;
  }
  __syncthreads();
  const bool ok = extend_plan(a, part, &bad);
  __threadfence_block();
  __syncthreads();
  extend_apply(a, ok, threadIdx.x, blockDim.x);
}

__global__ void __launch_bounds__(kPageThreads) extend_plan_kernel(ExtendArgs a) {
  __shared__ uint32_t part[17], bad;
  const bool ok = extend_plan(a, part, &bad);
  if (threadIdx.x == 0) *a.ok = ok;
}

__global__ void __launch_bounds__(256) extend_apply_kernel(ExtendArgs a) {
  extend_apply(a, *a.ok != 0u, blockIdx.x * blockDim.x + threadIdx.x, gridDim.x * blockDim.x);
}

// ------------------------------------------------------------------------------------------------ fork, trim
// A block per child: entries are copied as they are, each page's count goes up by one.
__global__ void __launch_bounds__(256) fork_kernel(PageArgs p, const int32_t* parents, const int32_t* children) {
  const uint32_t i = blockIdx.x;
  const int32_t from = parents[i], to = children[i];
  const bool inside = from >= 0 && (uint32_t)from < p.n_rows && to >= 0 && (uint32_t)to < p.n_rows;
  const int32_t held = inside ? p.length[from] : -1;
  const int64_t pages = ((int64_t)held + (1 << p.page_log2) - 1) >> p.page_log2;
  if (!inside || held < 0 || pages > p.width || p.length[to] != 0) {
    if (threadIdx.x == 0) raise(p.status, MAASO_INST_BAD_ROW);
    return;
  }
  for (uint32_t j = threadIdx.x; j < (uint32_t)pages; j += blockDim.x) {
    const int32_t page = p.table[(size_t)from * p.width + j];
    p.table[(size_t)to * p.width + j] = page;
    if (page >= 0 && (uint32_t)page < p.n_pages) atomicAdd(&p.refs[page], 1);
    else raise(p.status, MAASO_INST_BAD_PAGE);
  }
  __syncthreads();  // (every thread has read the child's length)
  if (threadIdx.x == 0) p.length[to] = held;
}

// A block per row: entries behind what is kept go, each page's count comes down by one.
__global__ void __launch_bounds__(256) trim_kernel(PageArgs p, const int32_t* rows, const int32_t* keep) {
  const uint32_t i = blockIdx.x;
  const int32_t row = rows[i], kept = keep[i];
  if (row < 0 || (uint32_t)row >= p.n_rows || kept < 0) {
    if (threadIdx.x == 0) raise(p.status, MAASO_INST_BAD_ROW);
    return;
  }
  const int32_t held = p.length[row];
  if (kept >= held) return;
  const int64_t per = 1 << p.page_log2;
  const int64_t begin = (kept + per - 1) >> p.page_log2, end = (held + per - 1) >> p.page_log2;
  if (end > p.width) {
    if (threadIdx.x == 0) raise(p.status, MAASO_INST_BAD_ROW);
    return;
  }
  for (int64_t j = begin + threadIdx.x; j < end; j += blockDim.x) {
    int32_t* at = &p.table[(size_t)row * p.width + (size_t)j];
    const int32_t page = *at;
    *at = -1;
    bool bad = page < 0 || (uint32_t)page >= p.n_pages;
    if (!bad && atomicSub(&p.refs[page], 1) <= 0) {
      atomicAdd(&p.refs[page], 1);
      bad = true;
    }
    if (bad) raise(p.status, MAASO_INST_BAD_PAGE);
  }
  __syncthreads();  // (every thread has read the length)
  if (threadIdx.x == 0) p.length[row] = kept;
}

// ------------------------------------------------------------------------------------------------ compact
// Held pages below p, `live(p)`, give every page's place: n_live is live(n_pages); a free page p < n_live is hole
// number p - live(p), a held page p >= n_live takes hole number live(p) - live(n_live).  Three launches: held pages
// of each chunk; live() of every page and the holes; the new numbers.  A pool of one chunk with a table that a block is
// through with at once, up to 32 entries a thread, takes one launch (3000 pages, 96 rows of 12, with the copy: 28 us, with one
// launch 21).
constexpr uint32_t kCompactChunk = 4096, kCompactEntries = 32 * kPageThreads;

struct CompactArgs {
  PageArgs p;
  int32_t* refs_out;
  int32_t* table_out;
  int32_t* moves;
  int32_t* n_live;
  // workspace
  uint32_t chunks;
  uint32_t* held;    // [chunks] held pages
  uint32_t* below;   // [n_pages + 1] live()
  int32_t* holes;    // [n_pages]
};

__global__ void __launch_bounds__(kPageThreads) compact_count_kernel(CompactArgs a) {
  __shared__ uint32_t part[17];
  const uint32_t p0 = blockIdx.x * kCompactChunk + threadIdx.x * 4u;
  uint32_t live = 0, sum;
  for (uint32_t k = 0; k < 4u; ++k)
    if (p0 + k < a.p.n_pages && a.p.refs[p0 + k] > 0) ++live;
  block_scan(live, part, sum);
  if (threadIdx.x == 0) a.held[blockIdx.x] = sum;
}

__device__ inline void compact_rank(const CompactArgs& a, uint32_t* part) {
  uint32_t before = 0, n_live = 0;
  for (uint32_t base = 0; a.chunks > 1u && base < a.chunks; base += blockDim.x) {
    const uint32_t c = base + threadIdx.x;
    const uint32_t v = c < a.chunks ? a.held[c] : 0u;
    uint32_t sum;
    block_scan(v, part, sum);
    n_live += sum;
    block_scan(c < blockIdx.x ? v : 0u, part, sum);
    before += sum;
  }
  const uint32_t p0 = blockIdx.x * kCompactChunk + threadIdx.x * 4u;
  uint32_t mine[4], live = 0, sum;
  for (uint32_t k = 0; k < 4u; ++k) {
    mine[k] = live;
    if (p0 + k < a.p.n_pages && a.p.refs[p0 + k] > 0) ++live;
    else mine[k] |= 0x80000000u;
  }
  const uint32_t at = before + block_scan(live, part, sum);
  if (a.chunks == 1u) n_live = sum;
  for (uint32_t k = 0; k < 4u; ++k) {
    const uint32_t p = p0 + k, r = at + (mine[k] & 0x7fffffffu);
    if (p < a.p.n_pages) {
      a.below[p] = r;
      if ((mine[k] >> 31) && p < n_live) a.holes[p - r] = (int32_t)p;
    }
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    a.below[a.p.n_pages] = n_live;
    *a.n_live = (int32_t)n_live;
  }
}

__device__ inline void compact_apply(const CompactArgs& a) {
  const uint32_t n = a.p.n_pages, n_live = a.below[n], low = a.below[n_live], threads = gridDim.x * blockDim.x;
  const uint32_t t = blockIdx.x * blockDim.x + threadIdx.x;
  const uint32_t moved = n_live - low;
  for (uint32_t p = t; p < n; p += threads) {
    const int32_t refs = a.p.refs[p];
    if (p < n_live) {
      if (refs > 0) a.refs_out[p] = refs;  // (a hole is written by the page that takes it)
    } else {
      if (refs > 0) {
        const uint32_t k = a.below[p] - low;
        const int32_t to = a.holes[k];
        a.refs_out[to] = refs;
        a.moves[2 * k] = (int32_t)p;
        a.moves[2 * k + 1] = to;
      }
      a.refs_out[p] = 0;
    }
    if (p < n / 2u && p >= moved) {
      a.moves[2 * p] = -1;
      a.moves[2 * p + 1] = -1;
    }
  }
  const uint64_t entries = (uint64_t)a.p.n_rows * a.p.width;
  for (uint64_t e = t; e < entries; e += threads) {
    int32_t p = a.p.table[e];
    if (p >= (int32_t)n || (p >= 0 && a.below[p + 1] == a.below[p])) {
      raise(a.p.status, MAASO_INST_BAD_PAGE);  // outside the pool, or held by the row and counted for nobody
      p = -1;
    } else if (p >= (int32_t)n_live) {
      p = a.holes[a.below[p] - low];
    } else if (p < 0) {
      p = -1;
    }
    a.table_out[e] = p;
  }
}

__global__ void __launch_bounds__(kPageThreads) compact_rank_kernel(CompactArgs a) {
  __shared__ uint32_t part[17];
  compact_rank(a, part);
}

__global__ void __launch_bounds__(256) compact_apply_kernel(CompactArgs a) { compact_apply(a); }

__global__ void __launch_bounds__(kPageThreads) compact_kernel(CompactArgs a) {
  __shared__ uint32_t part[17], below[kCompactChunk + 1];
  __shared__ int32_t holes[kCompactChunk];
  a.below = below;
  a.holes = holes;
  compact_rank(a, part);
  __syncthreads();
  compact_apply(a);
}

// ------------------------------------------------------------------------------------------------ copy
// Bound by memory: each block moves kCopyChunk bytes of a page, 16 bytes a thread, four loads ahead of the stores.  Pages of 32 KiB
// a layer packed 83 MB in and out in 15 us, faster than a large copy.  Copies that may be more than the L2s hold (32 MiB) are
// written past them: 48 copies of one page, 100 MB, with the calls around them 39 to 31 us; two copies of 1 MB 13.8 to 15.3.
constexpr uint64_t kCopyPast = 32u << 20;
constexpr uint32_t kCopyChunk = 16384;

struct CopyArgs {
  const int32_t* pairs;
  uint32_t n, n_pages, chunks, n_layers;
  uint64_t page_bytes, page_stride, layer_stride;  // bytes
  char* k;
  char* v;
  bool past;  // what is written goes past the caches
  uint32_t* status;
};

__global__ void __launch_bounds__(256) copy_kernel(CopyArgs a) {
  const uint32_t chunk = blockIdx.x % a.chunks, i = blockIdx.x / a.chunks, layer = blockIdx.y;
  const int32_t from = a.pairs[2 * (size_t)i], to = a.pairs[2 * (size_t)i + 1];
  if (from < 0 || to < 0) return;
  if ((uint32_t)from >= a.n_pages || (uint32_t)to >= a.n_pages) {
    if (threadIdx.x == 0 && chunk == 0 && layer == 0 && blockIdx.z == 0) raise(a.status, MAASO_INST_BAD_PAGE);
    return;
  }
  char* base = (blockIdx.z ? a.v : a.k) + layer * a.layer_stride;
  const uint64_t at = (uint64_t)chunk * kCopyChunk;
  const uint64_t left = a.page_bytes - at;
  typedef uint32_t piece __attribute__((ext_vector_type(4)));
  const piece* src = reinterpret_cast<const piece*>(base + (uint64_t)from * a.page_stride + at) + threadIdx.x;
  piece* dst = reinterpret_cast<piece*>(base + (uint64_t)to * a.page_stride + at) + threadIdx.x;
  if (left >= kCopyChunk) {
    const piece r0 = src[0], r1 = src[256], r2 = src[512], r3 = src[768];
    if (a.past) {
      keep_apart();
      __builtin_nontemporal_store(r0, dst);
      __builtin_nontemporal_store(r1, dst + 256);
      __builtin_nontemporal_store(r2, dst + 512);
      __builtin_nontemporal_store(r3, dst + 768);
      keep_apart();
    } else {
      dst[0] = r0;
      dst[256] = r1;
      dst[512] = r2;
      dst[768] = r3;
    }
  } else {
    for (uint32_t e = threadIdx.x; e < (uint32_t)left / 16u; e += 256u, src += 256, dst += 256) *dst = *src;
  }
}

}  // namespace maaso
