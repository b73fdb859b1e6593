// pages.hip - who holds which page of a paged cache (Section 6: fixed-size
// pages reached through block tables), kept on the device: counting, giving
// back, branching off, taking, compacting, and copying whole pages.
//
// Bookkeeping works on three small arrays (a count per page, the tables, the
// rows' lengths), so its time is launches and dependent reads, not bytes: a
// call is at most three launches, each a step whose input is the whole result
// of the one before (how much is wanted and how much is free; which pages;
// who gets them).  Every choice is "lowest free page first" by prefix sums,
// never by the order in which atomics land; atomics only add to counts, whose
// sum does not depend on the order.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "internal.h"
#include "topkv.h"

namespace topkv_pages {

constexpr int kThreads = 256;
constexpr int kPerThread = 16;                      // pages of one thread in a pass over the counts
constexpr int kPageBlock = kThreads * kPerThread;   // pages of one workgroup
constexpr int kMaxRows = TOPKV_MAX_BATCH_REQS;
constexpr int kMostRows = 1 << 22;                  // of an owner: a launch holds fewer than 2^32 threads

// Workspace, in int32 words: [0] the rows are good, [1] pages wanted, [2] the
// call goes ahead, then per row of the call: first page of its share, first
// pair, its old length; then per row of the owner a mark that finds rows
// named twice; then free (or live) pages per block; then a word per page
// (pages taken in order, or a moving page's pair).
struct Work {
  int32_t* head;
  int32_t* page_at;
  int32_t* pair_at;
  int32_t* old_len;
  int32_t* mark;
  int32_t* block;
  int32_t* page;
};

int64_t blocks_of(int64_t num_pages) { return (num_pages + kPageBlock - 1) / kPageBlock; }

int64_t work_words(const topkv_page_owner_t* o) {
  const int64_t per_call = o->num_rows < kMaxRows ? o->num_rows : kMaxRows;
  return 16 + 3 * per_call + o->num_rows + blocks_of(o->num_pages) + o->num_pages;
}

Work carve(const topkv_page_owner_t* o, void* workspace) {
  const int64_t per_call = o->num_rows < kMaxRows ? o->num_rows : kMaxRows;
  Work w;
  w.head = static_cast<int32_t*>(workspace);
  w.page_at = w.head + 16;
  w.pair_at = w.page_at + per_call;
  w.old_len = w.pair_at + per_call;
  w.mark = w.old_len + per_call;
  w.block = w.mark + o->num_rows;
  w.page = w.block + blocks_of(o->num_pages);
  return w;
}

__device__ __forceinline__ int32_t pages_for(int32_t tokens, int32_t page_size) {
  return (int32_t)(((int64_t)tokens + page_size - 1) / page_size);
}

// Sum over the workgroup, returned to every thread (s: one word per wave, a
// different array for every call of a kernel).
template <class I>
__device__ __forceinline__ I block_sum(I v, I* s) {
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d, 64);
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  I t = 0;
  for (int i = 0; i < kThreads / 64; ++i) t += s[i];
  return t;
}

// Exclusive prefix sum over the workgroup's threads, and the sum.
template <class I>
__device__ __forceinline__ I block_scan(I v, I* s, I* total) {
  I inc = v;
  const int lane = threadIdx.x & 63;
  for (int d = 1; d < 64; d <<= 1) {
    const I up = __shfl_up(inc, d, 64);
    if (lane >= d) inc += up;
  }
  if (lane == 63) s[threadIdx.x >> 6] = inc;
  __syncthreads();
  I before = 0, all = 0;
  for (int i = 0; i < kThreads / 64; ++i) {
    if (i < (int)(threadIdx.x >> 6)) before += s[i];
    all += s[i];
  }
  *total = all;
  return before + inc - v;
}

// Bit i: page first + i exists and is live (count above 0).
__device__ __forceinline__ uint32_t live_bits(const int32_t* __restrict__ refs, int64_t first, int64_t num_pages) {
  uint32_t bits = 0;
#pragma unroll
  for (int i = 0; i < kPerThread; ++i) {
    const int64_t p = first + i;
    const int32_t c = refs[p < num_pages ? p : num_pages - 1];
    bits |= (uint32_t)(p < num_pages && c > 0) << i;
  }
  return bits;
}

__device__ __forceinline__ uint32_t page_bits(int64_t first, int64_t num_pages) {
  const int64_t left = num_pages - first;
  return left >= kPerThread ? (1u << kPerThread) - 1 : left > 0 ? (1u << left) - 1 : 0;
}

// Live and all pages before this workgroup's, and live pages in all.
__device__ void block_prefix(const int32_t* __restrict__ live, int32_t blocks, int32_t mine, int32_t (*s)[kThreads / 64],
                             int32_t* before, int32_t* total) {
  int32_t b = 0, t = 0;
  for (int32_t i = threadIdx.x; i < blocks; i += kThreads) {
    const int32_t v = live[i];
    t += v;
    if (i < mine) b += v;
  }
  *before = block_sum(b, s[0]);
  *total = block_sum(t, s[1]);
}

// Looks the rows of a fork or grow over, adds up what they want and sets the
// result words; one workgroup.  *ok, *all_want: for every thread.
template <bool kFork>
__device__ void plan_rows(const topkv_page_owner_t& o, int32_t num, const int32_t* __restrict__ a,
                          const int32_t* __restrict__ b, const Work& w, int32_t* __restrict__ result, bool* good,
                          int64_t* all_want) {
  __shared__ int64_t s_want[kThreads / 64];
  __shared__ uint32_t s_rest[kThreads / 64];
  const int32_t cap = o.bt_stride * o.page_size;
  const int32_t* rows = kFork ? b : a;               // the rows that get pages
  for (int32_t i = threadIdx.x; i < num; i += kThreads) {
    const int32_t row = rows[i];
    if (row >= 0 && row < o.num_rows) __hip_atomic_store(&w.mark[row], i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __threadfence();
  __syncthreads();
  // The last naming of a row is the good one.  Which store came last is chance: where a row has another's mark the
  // highest number is found, so that the count of bad rows does not depend on it.
  bool other = false;
  for (int32_t i = threadIdx.x; i < num; i += kThreads) {
    const int32_t row = rows[i];
    if (row >= 0 && row < o.num_rows)
      other |= __hip_atomic_load(&w.mark[row], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != i;
  }
  if (__syncthreads_or(other)) {
    for (int32_t i = threadIdx.x; i < num; i += kThreads) {
      const int32_t row = rows[i];
      if (row >= 0 && row < o.num_rows) atomicMax(&w.mark[row], i);
    }
    __threadfence();
    __syncthreads();
  }
  const int32_t per = (num + kThreads - 1) / kThreads;
  const int32_t lo = threadIdx.x * per, hi = lo + per < num ? lo + per : num;
  int64_t want = 0;
  uint32_t rest = 0;                                 // pairs, and bad rows from bit 16 on: at most kMaxRows of either
  for (int32_t i = lo; i < hi; ++i) {
    const int32_t row = rows[i];
    int32_t need = 0, pair = 0, old = 0;
    bool ok = row >= 0 && row < o.num_rows &&
              __hip_atomic_load(&w.mark[row], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == i;
    if (kFork) {
      const int32_t par = a[i];
      ok = ok && par >= 0 && par < o.num_rows && o.seq_lens[row] == 0;
      if (ok) {
        old = o.seq_lens[par];
        ok = old >= 0 && old <= cap;
        need = pair = ok && old % o.page_size != 0;
      }
    } else if (ok) {
      const int32_t upto = b[i];
      old = o.seq_lens[row];
      ok = old >= 0 && upto >= old && upto <= cap;
      if (ok) {
        need = pages_for(upto, o.page_size) - pages_for(old, o.page_size);
        if (upto > old && old % o.page_size != 0) {
          const int32_t e = o.block_tables[(int64_t)row * o.bt_stride + old / o.page_size];
          if (e >= 0 && e < o.num_pages && o.ref_counts[e] > 1) pair = 1;
          need += pair;
        }
      }
    }
    rest += (uint32_t)pair | (uint32_t)!ok << 16;
    w.page_at[i] = need;
    w.pair_at[i] = pair;
    w.old_len[i] = old;
    want += need;
  }
  int64_t all;
  uint32_t all_rest;
  int64_t at = block_scan(want, s_want, &all);
  int32_t pair_at = (int32_t)(block_scan(rest, s_rest, &all_rest) & 0xffffu);
  const int32_t all_pairs = (int32_t)(all_rest & 0xffffu), all_bad = (int32_t)(all_rest >> 16);
  for (int32_t i = lo; i < hi; ++i) {                // a share past 2^31 is more than any pool has: never used
    const int32_t need = w.page_at[i], pair = w.pair_at[i];
    w.page_at[i] = (int32_t)at;
    w.pair_at[i] = pair_at;
    at += need;
    pair_at += pair;
  }
  *good = all_bad == 0;
  *all_want = all;
  if (threadIdx.x == 0) {
    w.head[0] = all_bad == 0;
    w.head[1] = (int32_t)(all < INT32_MAX ? all : INT32_MAX);
    result[0] = all_bad ? TOPKV_ERR_BOUNDS : TOPKV_OK;
    result[1] = all_bad ? 0 : all_pairs;
    result[2] = w.head[1];
    result[3] = all_bad;
  }
}

// Whether the call goes ahead (thread 0 of one workgroup).
__device__ __forceinline__ void verdict(const Work& w, bool ahead, int32_t* __restrict__ result) {
  w.head[2] = ahead;
  if (!ahead) {
    result[0] = TOPKV_ERR_BOUNDS;
    result[1] = 0;
  }
}

// This thread's free pages (bits from page `first` on, the lowest one number
// `rank` of all free pages), those wanted into w.page with a count of 1.
__device__ __forceinline__ void take_pages(const topkv_page_owner_t& o, const Work& w, uint32_t free_bits, int64_t first,
                                           int64_t rank, int64_t want) {
  for (; free_bits && rank < want; free_bits &= free_bits - 1, ++rank) {
    const int32_t p = (int32_t)(first + __ffs(free_bits) - 1);
    w.page[rank] = p;
    o.ref_counts[p] = 1;
  }
}

// Step 1 of fork and grow: workgroup 0 plans the rows, workgroup 1 + b counts
// the live pages of block b.
template <bool kFork>
__global__ __launch_bounds__(kThreads) void kv_pages_plan_kernel(topkv_page_owner_t o, int32_t num,
                                                                 const int32_t* __restrict__ a,
                                                                 const int32_t* __restrict__ b, Work w,
                                                                 int32_t* __restrict__ result) {
  __shared__ int32_t s[kThreads / 64];
  if (blockIdx.x > 0) {
    const int64_t first = ((int64_t)(blockIdx.x - 1) * kThreads + threadIdx.x) * kPerThread;
    const int32_t n = block_sum((int32_t)__popc(live_bits(o.ref_counts, first, o.num_pages)), s);
    if (threadIdx.x == 0) w.block[blockIdx.x - 1] = n;
    return;
  }
  bool ok;
  int64_t want;
  plan_rows<kFork>(o, num, a, b, w, result, &ok, &want);
}

// Step 2: the wanted number of free pages, lowest first, in w.page.
__global__ __launch_bounds__(kThreads) void kv_pages_take_kernel(topkv_page_owner_t o, Work w, int32_t blocks,
                                                                 int32_t* __restrict__ result) {
  __shared__ int32_t s[3][kThreads / 64];
  int32_t live_before, live, in_block;
  block_prefix(w.block, blocks, blockIdx.x, s, &live_before, &live);
  const int64_t want = w.head[1];
  const bool ahead = w.head[0] && want <= o.num_pages - live;
  if (blockIdx.x == 0 && threadIdx.x == 0) verdict(w, ahead, result);
  const int64_t rank = (int64_t)blockIdx.x * kPageBlock - live_before;      // free pages before this block
  if (!ahead || rank >= want) return;
  const int64_t first = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * kPerThread;
  const uint32_t free_bits = ~live_bits(o.ref_counts, first, o.num_pages) & page_bits(first, o.num_pages);
  take_pages(o, w, free_bits, first, rank + block_scan((int32_t)__popc(free_bits), s[2], &in_block), want);
}

// Steps 1 and 2 in one workgroup, for pools of few blocks (1300 pages, 128
// rows: a launch less, 75.5 -> 73.4 us for a beam step of two such calls).
constexpr int kFewBlocks = 4;

template <bool kFork>
__global__ __launch_bounds__(kThreads) void kv_pages_plan_take_kernel(topkv_page_owner_t o, int32_t num,
                                                                      const int32_t* __restrict__ a,
                                                                      const int32_t* __restrict__ b, Work w,
                                                                      int32_t* __restrict__ result) {
  __shared__ uint64_t s[kThreads / 64];
  uint32_t free_bits[kFewBlocks];
  uint64_t counts = 0, all;                          // 16 bits a block
#pragma unroll
  for (int k = 0; k < kFewBlocks; ++k) {
    const int64_t first = ((int64_t)k * kThreads + threadIdx.x) * kPerThread;
    free_bits[k] = ~live_bits(o.ref_counts, first, o.num_pages) & page_bits(first, o.num_pages);
    counts |= (uint64_t)__popc(free_bits[k]) << (16 * k);
  }
  const uint64_t before = block_scan(counts, s, &all);
  bool ok;
  int64_t want, room = 0;
  plan_rows<kFork>(o, num, a, b, w, result, &ok, &want);
#pragma unroll
  for (int k = 0; k < kFewBlocks; ++k) room += all >> (16 * k) & 0xffffu;
  const bool ahead = room >= want && ok;
  if (threadIdx.x == 0) verdict(w, ahead, result);
  if (!ahead) return;
  int64_t rank = 0;
#pragma unroll
  for (int k = 0; k < kFewBlocks; ++k) {
    take_pages(o, w, free_bits[k], ((int64_t)k * kThreads + threadIdx.x) * kPerThread, rank + (before >> (16 * k) & 0xffffu),
               want);
    rank += all >> (16 * k) & 0xffffu;
  }
}

// Step 3 of fork: one workgroup per child.
__global__ __launch_bounds__(kThreads) void kv_pages_fork_kernel(topkv_page_owner_t o,
                                                                 const int32_t* __restrict__ parents,
                                                                 const int32_t* __restrict__ children, Work w,
                                                                 int32_t* __restrict__ pairs,
                                                                 int32_t* __restrict__ result) {
  if (!w.head[2]) return;
  const int32_t i = blockIdx.x, n = w.old_len[i], whole = n / o.page_size;
  const int32_t* from = o.block_tables + (int64_t)parents[i] * o.bt_stride;
  int32_t* to = o.block_tables + (int64_t)children[i] * o.bt_stride;
  int32_t bad = 0;
  for (int32_t j = threadIdx.x; j < whole; j += kThreads) {
    const int32_t e = from[j];
    to[j] = e;
    if (e >= 0 && e < o.num_pages) atomicAdd(&o.ref_counts[e], 1);
    else ++bad;
  }
  if (threadIdx.x == 0) {
    if (n % o.page_size != 0) {
      const int32_t p = w.page[w.page_at[i]], e = from[whole];
      to[whole] = p;
      pairs[2 * w.pair_at[i]] = e;
      pairs[2 * w.pair_at[i] + 1] = p;
      bad += e < 0 || e >= o.num_pages;
    }
    o.seq_lens[children[i]] = n;
  }
  if (bad) {
    atomicAdd(&result[3], bad);
    result[0] = TOPKV_ERR_BOUNDS;
  }
}

// Step 3 of grow: one workgroup per row.
__global__ __launch_bounds__(kThreads) void kv_pages_grow_kernel(topkv_page_owner_t o, int32_t num,
                                                                 const int32_t* __restrict__ rows,
                                                                 const int32_t* __restrict__ new_lens, Work w,
                                                                 int32_t* __restrict__ pairs,
                                                                 const int32_t* __restrict__ result) {
  if (!w.head[2]) return;
  const int32_t i = blockIdx.x, old = w.old_len[i], upto = new_lens[i];
  const int32_t have = pages_for(old, o.page_size), need = pages_for(upto, o.page_size) - have;
  const int32_t all_pairs = result[1];
  const int32_t pair = (i + 1 < num ? w.pair_at[i + 1] : all_pairs) - w.pair_at[i];
  int32_t* row = o.block_tables + (int64_t)rows[i] * o.bt_stride;
  const int32_t at = w.page_at[i];
  if (threadIdx.x == 0) {
    if (pair) {
      const int32_t e = row[have - 1], p = w.page[at];
      row[have - 1] = p;
      pairs[2 * w.pair_at[i]] = e;
      pairs[2 * w.pair_at[i] + 1] = p;
      atomicSub(&o.ref_counts[e], 1);
    }
    o.seq_lens[rows[i]] = upto;
  }
  for (int32_t j = threadIdx.x; j < need; j += kThreads) row[have + j] = w.page[at + pair + j];
}

__global__ void kv_pages_begin_kernel(int32_t* __restrict__ result) {
  if (threadIdx.x < 4) result[threadIdx.x] = 0;
}

// Give back: one workgroup per named row.  The exchange hands each entry to
// one thread only, so a row named twice gives every page back once.  The other
// workgroup may lower the row's length at any time: one thread reads it, for all.
__global__ __launch_bounds__(kThreads) void kv_pages_free_kernel(topkv_page_owner_t o, const int32_t* __restrict__ rows,
                                                                 const int32_t* __restrict__ keep_lens,
                                                                 int32_t* __restrict__ result) {
  __shared__ int32_t s_len;
  const int32_t row = rows[blockIdx.x];
  const int32_t keep = keep_lens ? keep_lens[blockIdx.x] : 0;
  if (threadIdx.x == 0)
    s_len = row < 0 || row >= o.num_rows || keep < 0
                ? -1
                : __hip_atomic_load(&o.seq_lens[row], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  const int32_t n = s_len;
  int32_t bad = 0, gone = 0;
  if (n < 0 || n > o.bt_stride * o.page_size) {
    bad = threadIdx.x == 0;
  } else if (keep < n) {
    int32_t* tab = o.block_tables + (int64_t)row * o.bt_stride;
    const int32_t held = pages_for(n, o.page_size);
    for (int32_t j = pages_for(keep, o.page_size) + threadIdx.x; j < held; j += kThreads) {
      const int32_t e = atomicExch(&tab[j], -1);
      if (e == -1) continue;                                         // given back already
      if (e < 0 || e >= o.num_pages) {
        ++bad;
      } else if (atomicSub(&o.ref_counts[e], 1) <= 0) {
        atomicAdd(&o.ref_counts[e], 1);
        ++bad;
      } else {
        ++gone;
      }
    }
    if (threadIdx.x == 0) atomicMin(&o.seq_lens[row], keep);
  }
  if (gone) atomicAdd(&result[2], gone);
  if (bad) {
    atomicAdd(&result[3], bad);
    result[0] = TOPKV_ERR_BOUNDS;
  }
}

__global__ __launch_bounds__(kThreads) void kv_pages_clear_kernel(int32_t* __restrict__ refs, int64_t num_pages,
                                                                  int32_t* __restrict__ result) {
  const int64_t step = (int64_t)gridDim.x * kThreads;
  for (int64_t p = (int64_t)blockIdx.x * kThreads + threadIdx.x; p < num_pages; p += step) refs[p] = 0;
  if (blockIdx.x == 0 && threadIdx.x < 4) result[threadIdx.x] = 0;
}

__global__ __launch_bounds__(kThreads) void kv_pages_count_kernel(topkv_page_owner_t o, int32_t* __restrict__ result) {
  const int32_t row = blockIdx.x, n = o.seq_lens[row];
  int32_t bad = 0, named = 0;
  if (n < 0 || n > o.bt_stride * o.page_size) {
    bad = threadIdx.x == 0;
  } else {
    const int32_t held = pages_for(n, o.page_size);
    for (int32_t j = threadIdx.x; j < held; j += kThreads) {
      const int32_t e = o.block_tables[(int64_t)row * o.bt_stride + j];
      if (e < 0 || e >= o.num_pages) {
        ++bad;
      } else {
        named += atomicAdd(&o.ref_counts[e], 1) == 0;                // first to name it
      }
    }
  }
  if (named) atomicAdd(&result[2], named);
  if (bad) {
    atomicAdd(&result[3], bad);
    result[0] = TOPKV_ERR_BOUNDS;
  }
}

// Compaction, step 1: live pages per block.
__global__ __launch_bounds__(kThreads) void kv_pages_live_kernel(topkv_page_owner_t o, Work w,
                                                                 int32_t* __restrict__ result) {
  __shared__ int32_t s[kThreads / 64];
  const int64_t first = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * kPerThread;
  const int32_t n = block_sum((int32_t)__popc(live_bits(o.ref_counts, first, o.num_pages)), s);
  if (threadIdx.x == 0) w.block[blockIdx.x] = n;
  if (blockIdx.x == 0 && threadIdx.x < 4) result[threadIdx.x] = 0;
}

// Step 2: with U live pages, free page p < U is hole number (free pages
// before p); live page p >= U is mover number (live pages after p).  Hole and
// mover of one number make a pair.
__global__ __launch_bounds__(kThreads) void kv_pages_match_kernel(topkv_page_owner_t o, Work w, int32_t blocks,
                                                                  int32_t* __restrict__ pairs,
                                                                  int32_t* __restrict__ result) {
  __shared__ int32_t s[3][kThreads / 64];
  int32_t before, live, in_block;
  block_prefix(w.block, blocks, blockIdx.x, s, &before, &live);
  const int64_t first = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * kPerThread;
  const uint32_t bits = live_bits(o.ref_counts, first, o.num_pages);
  before += block_scan((int32_t)__popc(bits), s[2], &in_block);
  if (blockIdx.x == 0 && threadIdx.x == 0) result[2] = live;
  for (int i = 0; i < kPerThread && first + i < o.num_pages; ++i) {
    const int64_t p = first + i, prior = before + __popc(bits & ((1u << i) - 1));
    const bool is_live = bits >> i & 1;
    if (p == live) result[1] = (int32_t)(live - prior);              // movers in all
    if (!is_live && p < live) pairs[2 * (p - prior) + 1] = (int32_t)p;
    if (is_live && p >= live) {
      const int64_t k = live - prior - 1;
      pairs[2 * k] = (int32_t)p;
      w.page[p] = (int32_t)k;
    }
  }
}

// Step 3: workgroup r < num_rows renames the entries of row r, the others
// move the counts.
__global__ __launch_bounds__(kThreads) void kv_pages_rename_kernel(topkv_page_owner_t o, Work w,
                                                                   const int32_t* __restrict__ pairs,
                                                                   int32_t* __restrict__ result) {
  const int32_t moved = result[1], live = result[2];
  if ((int64_t)blockIdx.x >= o.num_rows) {
    const int32_t step = (int32_t)(gridDim.x - o.num_rows) * kThreads;
    for (int64_t k = (int64_t)(blockIdx.x - o.num_rows) * kThreads + threadIdx.x; k < moved; k += step) {
      const int32_t src = pairs[2 * k], dst = pairs[2 * k + 1];
      o.ref_counts[dst] = o.ref_counts[src];
      o.ref_counts[src] = 0;
    }
    return;
  }
  const int32_t n = o.seq_lens[blockIdx.x];
  int32_t bad = 0;
  if (n < 0 || n > o.bt_stride * o.page_size) {
    bad = threadIdx.x == 0;
  } else {
    int32_t* tab = o.block_tables + (int64_t)blockIdx.x * o.bt_stride;
    const int32_t held = pages_for(n, o.page_size);
    for (int32_t j = threadIdx.x; j < held; j += kThreads) {
      const int32_t e = tab[j];
      if (e < 0 || e >= o.num_pages) {
        ++bad;
      } else if (e >= live) {
        const int32_t k = w.page[e];
        if (k >= 0 && k < moved && pairs[2 * k] == e) tab[j] = pairs[2 * k + 1];
        else ++bad;                                                  // names a free page
      }
    }
  }
  if (bad) {
    atomicAdd(&result[3], bad);
    result[0] = TOPKV_ERR_BOUNDS;
  }
}

// ---- whole pages -------------------------------------------------------------
template <int B> struct Vec;
template <> struct Vec<16> { typedef unsigned int type __attribute__((ext_vector_type(4))); };
template <> struct Vec<4> { typedef unsigned int type; };
template <> struct Vec<1> { typedef unsigned char type; };

struct CopyParams {
  int64_t src_pages, dst_pages, page_bytes;
  int64_t src_layer, dst_layer;    // bytes of a layer
  int32_t tiles;                   // of a page
  int32_t max_pairs;
};

// A page of a layer is one contiguous run on both sides.  grid.x strides over
// (pair, tile of the page), grid.y is the layer; all loads of a tile are
// issued before its stores.
template <int VB, int VPT>
__global__ __launch_bounds__(kThreads) void kv_copy_pages_kernel(const char* __restrict__ src, char* __restrict__ dst,
                                                                 const int32_t* __restrict__ pairs,
                                                                 const int32_t* __restrict__ count, CopyParams p) {
  typedef typename Vec<VB>::type V;
  constexpr int kTile = kThreads * VPT;              // vectors
  int32_t n = p.max_pairs;
  if (count) {
    n = *count;
    n = n < 0 ? 0 : n > p.max_pairs ? p.max_pairs : n;
  }
  const uint32_t items = (uint32_t)n * (uint32_t)p.tiles;
  src += (int64_t)blockIdx.y * p.src_layer;
  dst += (int64_t)blockIdx.y * p.dst_layer;
  const int64_t vectors = p.page_bytes / VB;
  for (uint32_t it = blockIdx.x; it < items; it += gridDim.x) {
    const uint32_t k = it / (uint32_t)p.tiles, tile = it - k * (uint32_t)p.tiles;
    const int32_t s = pairs[2 * (int64_t)k], d = pairs[2 * (int64_t)k + 1];
    if (s < 0 || s >= p.src_pages || d < 0 || d >= p.dst_pages) continue;
    const V* from = reinterpret_cast<const V*>(src + s * p.page_bytes) + (int64_t)tile * kTile;
    V* to = reinterpret_cast<V*>(dst + d * p.page_bytes) + (int64_t)tile * kTile;
    const int64_t left = vectors - (int64_t)tile * kTile;
    V v[VPT];
    if (left >= kTile) {
#pragma unroll
      for (int j = 0; j < VPT; ++j) v[j] = __builtin_nontemporal_load(from + j * kThreads + threadIdx.x);
#pragma unroll
      for (int j = 0; j < VPT; ++j) __builtin_nontemporal_store(v[j], to + j * kThreads + threadIdx.x);
    } else {
      const int32_t nv = (int32_t)left;
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        const int x = j * kThreads + (int)threadIdx.x;
        v[j] = from[x < nv ? x : nv - 1];
      }
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        const int x = j * kThreads + (int)threadIdx.x;
        if (x < nv) to[x] = v[j];
      }
    }
  }
}

topkv_status_t launched() { return hipGetLastError() == hipSuccess ? TOPKV_OK : TOPKV_ERR_LAUNCH; }

bool owner_ok(const topkv_page_owner_t* o) {
  return o && o->ref_counts && o->block_tables && o->seq_lens && o->num_pages > 0 && o->num_pages < INT32_MAX &&
         o->page_size > 0 && o->num_rows > 0 && o->num_rows <= kMostRows && o->bt_stride > 0 && o->reserved == 0 &&
         (int64_t)o->bt_stride * o->page_size <= INT32_MAX;
}

bool work_ok(const topkv_page_owner_t* o, const void* workspace, int64_t bytes) {
  return workspace && reinterpret_cast<uintptr_t>(workspace) % 16 == 0 && bytes >= 4 * work_words(o);
}

template <bool kFork>
topkv_status_t take(const topkv_page_owner_t* o, int32_t num, const int32_t* a, const int32_t* b, int32_t* pairs,
                    int32_t max_pairs, void* workspace, int64_t workspace_bytes, int32_t* result, hipStream_t stream) {
  if (!owner_ok(o) || num < 0 || num > kMaxRows || num > o->num_rows || !result || !work_ok(o, workspace, workspace_bytes))
    return TOPKV_ERR_INVALID_ARG;
  if (num > 0 && (!a || !b || !pairs || max_pairs < num)) return TOPKV_ERR_INVALID_ARG;
  if (num == 0) {
    hipLaunchKernelGGL(kv_pages_begin_kernel, dim3(1), dim3(64), 0, stream, result);
    return launched();
  }
  const Work w = carve(o, workspace);
  const int32_t blocks = (int32_t)blocks_of(o->num_pages);
  if (blocks <= kFewBlocks) {
    hipLaunchKernelGGL(HIP_KERNEL_NAME(kv_pages_plan_take_kernel<kFork>), dim3(1), dim3(kThreads), 0, stream, *o, num, a, b, w,
                       result);
  } else {
    hipLaunchKernelGGL(HIP_KERNEL_NAME(kv_pages_plan_kernel<kFork>), dim3(1 + blocks), dim3(kThreads), 0, stream, *o, num, a,
                       b, w, result);
    if (launched() != TOPKV_OK) return TOPKV_ERR_LAUNCH;
    hipLaunchKernelGGL(kv_pages_take_kernel, dim3(blocks), dim3(kThreads), 0, stream, *o, w, blocks, result);
  }
  if (launched() != TOPKV_OK) return TOPKV_ERR_LAUNCH;
  if (kFork)
    hipLaunchKernelGGL(kv_pages_fork_kernel, dim3(num), dim3(kThreads), 0, stream, *o, a, b, w, pairs, result);
  else
    hipLaunchKernelGGL(kv_pages_grow_kernel, dim3(num), dim3(kThreads), 0, stream, *o, num, a, b, w, pairs, result);
  return launched();
}

}  // namespace topkv_pages

extern "C" {

using namespace topkv_pages;

int64_t topkv_pages_workspace_bytes(const topkv_page_owner_t* owner) {
  return owner_ok(owner) ? 4 * work_words(owner) : -1;
}

topkv_status_t topkv_pages_count(const topkv_page_owner_t* owner, int32_t* result, hipStream_t stream) {
  if (!owner_ok(owner) || !result) return TOPKV_ERR_INVALID_ARG;
  const int64_t need = (owner->num_pages + kThreads - 1) / kThreads;
  hipLaunchKernelGGL(kv_pages_clear_kernel, dim3((unsigned)(need < 1024 ? need : 1024)), dim3(kThreads), 0, stream,
                     owner->ref_counts, owner->num_pages, result);
  if (launched() != TOPKV_OK) return TOPKV_ERR_LAUNCH;
  hipLaunchKernelGGL(kv_pages_count_kernel, dim3(owner->num_rows), dim3(kThreads), 0, stream, *owner, result);
  return launched();
}

topkv_status_t topkv_pages_free(const topkv_page_owner_t* owner, int32_t num, const int32_t* rows,
                                const int32_t* keep_lens, int32_t* result, hipStream_t stream) {
  if (!owner_ok(owner) || num < 0 || num > kMaxRows || !result || (num > 0 && !rows)) return TOPKV_ERR_INVALID_ARG;
  hipLaunchKernelGGL(kv_pages_begin_kernel, dim3(1), dim3(64), 0, stream, result);
  if (launched() != TOPKV_OK || num == 0) return launched();
  hipLaunchKernelGGL(kv_pages_free_kernel, dim3(num), dim3(kThreads), 0, stream, *owner, rows, keep_lens, result);
  return launched();
}

topkv_status_t topkv_pages_fork(const topkv_page_owner_t* owner, int32_t num, const int32_t* parents,
                                const int32_t* children, int32_t* pairs, int32_t max_pairs, void* workspace,
                                int64_t workspace_bytes, int32_t* result, hipStream_t stream) {
  return take<true>(owner, num, parents, children, pairs, max_pairs, workspace, workspace_bytes, result, stream);
}

topkv_status_t topkv_pages_grow(const topkv_page_owner_t* owner, int32_t num, const int32_t* rows,
                                const int32_t* new_lens, int32_t* pairs, int32_t max_pairs, void* workspace,
                                int64_t workspace_bytes, int32_t* result, hipStream_t stream) {
  return take<false>(owner, num, rows, new_lens, pairs, max_pairs, workspace, workspace_bytes, result, stream);
}

topkv_status_t topkv_pages_compact(const topkv_page_owner_t* owner, int32_t* pairs, int32_t max_pairs,
                                   void* workspace, int64_t workspace_bytes, int32_t* result, hipStream_t stream) {
  if (!owner_ok(owner) || !result || !work_ok(owner, workspace, workspace_bytes)) return TOPKV_ERR_INVALID_ARG;
  if (max_pairs < owner->num_pages / 2 || (!pairs && owner->num_pages > 1)) return TOPKV_ERR_INVALID_ARG;
  const Work w = carve(owner, workspace);
  const int32_t blocks = (int32_t)blocks_of(owner->num_pages);
  hipLaunchKernelGGL(kv_pages_live_kernel, dim3(blocks), dim3(kThreads), 0, stream, *owner, w, result);
  if (launched() != TOPKV_OK) return TOPKV_ERR_LAUNCH;
  hipLaunchKernelGGL(kv_pages_match_kernel, dim3(blocks), dim3(kThreads), 0, stream, *owner, w, blocks, pairs, result);
  if (launched() != TOPKV_OK) return TOPKV_ERR_LAUNCH;
  const int64_t movers = (owner->num_pages / 2 + kThreads - 1) / kThreads;
  const int64_t extra = movers < 1 ? 1 : movers < 256 ? movers : 256;
  hipLaunchKernelGGL(kv_pages_rename_kernel, dim3((unsigned)(owner->num_rows + extra)), dim3(kThreads), 0, stream, *owner, w,
                     pairs, result);
  return launched();
}

topkv_status_t topkv_copy_pages(const topkv_pool_t* src, const topkv_pool_t* dst, int32_t first_layer,
                                int32_t num_layers, const int32_t* pairs, int32_t max_pairs, const int32_t* count,
                                hipStream_t stream) {
  if (!src || !dst) return TOPKV_ERR_INVALID_ARG;
  topkv_status_t st = topkv_internal::pool_ok(src);
  if (st == TOPKV_OK) st = topkv_internal::pool_ok(dst);
  if (st != TOPKV_OK) return st;
  if (src->planes != dst->planes || src->page_size != dst->page_size || src->num_heads != dst->num_heads ||
      src->head_dim != dst->head_dim || src->elem_bytes != dst->elem_bytes)
    return TOPKV_ERR_INVALID_ARG;
  if (first_layer < 0 || num_layers < 0 || max_pairs < 0 || (int64_t)first_layer + num_layers > src->num_layers ||
      (int64_t)first_layer + num_layers > dst->num_layers)
    return TOPKV_ERR_INVALID_ARG;
  if (num_layers == 0 || max_pairs == 0) return TOPKV_OK;
  if (!pairs) return TOPKV_ERR_INVALID_ARG;
  CopyParams p;
  p.src_pages = src->num_pages;
  p.dst_pages = dst->num_pages;
  p.page_bytes = (int64_t)src->planes * src->page_size * src->num_heads * src->head_dim * src->elem_bytes;
  p.src_layer = p.page_bytes * src->num_pages;
  p.dst_layer = p.page_bytes * dst->num_pages;
  p.max_pairs = max_pairs;
  const char* from = static_cast<const char*>(src->base) + first_layer * p.src_layer;
  char* to = static_cast<char*>(dst->base) + first_layer * p.dst_layer;
  const uintptr_t all = reinterpret_cast<uintptr_t>(from) | reinterpret_cast<uintptr_t>(to) | (uintptr_t)p.page_bytes;
  const int vb = all % 16 == 0 ? 16 : all % 4 == 0 ? 4 : 1;
  int vpt = 8;
  while (vpt > 1 && (int64_t)kThreads * (vpt / 2) * vb >= p.page_bytes) vpt >>= 1;
  const int64_t tile = (int64_t)kThreads * vpt * vb, tiles = (p.page_bytes + tile - 1) / tile;
  if (tiles * max_pairs > INT32_MAX || num_layers > 65535) return TOPKV_ERR_UNSUPPORTED;
  p.tiles = (int32_t)tiles;
  const int64_t share = (16384 + num_layers - 1) / num_layers, items = tiles * max_pairs;
  const dim3 grid((unsigned)(items < share ? items : share), (unsigned)num_layers);
#define TOPKV_COPY(VB, VPT) \
  hipLaunchKernelGGL(HIP_KERNEL_NAME(kv_copy_pages_kernel<VB, VPT>), grid, dim3(kThreads), 0, stream, from, to, pairs, count, p)
#define TOPKV_COPY_VB(VB)                  \
  do {                                     \
    if (vpt == 8) TOPKV_COPY(VB, 8);       \
    else if (vpt == 4) TOPKV_COPY(VB, 4);  \
    else if (vpt == 2) TOPKV_COPY(VB, 2);  \
    else TOPKV_COPY(VB, 1);                \
  } while (0)
  if (vb == 16) TOPKV_COPY_VB(16);
  else if (vb == 4) TOPKV_COPY_VB(4);
  else TOPKV_COPY_VB(1);
#undef TOPKV_COPY_VB
#undef TOPKV_COPY
  return launched();
}

}  // extern "C"
