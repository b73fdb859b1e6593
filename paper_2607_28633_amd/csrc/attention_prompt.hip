// attention_prompt.hip - many new tokens per request on the matrix units.
//
// A workgroup takes 128 or 256 query rows of one KV head, a row being one
// (token, query head of the group): neighbouring tokens and all heads of the
// group read the same keys, so even a short chunk fills the rows.  Four or
// eight waves of 32 rows walk tiles of 64 keys: scores^T = K Q^T, running maximum and sum,
// out^T += V^T P^T, 4 * 32 * 64 * head_dim flops a wave and tile against
// 256 * head_dim bytes of LDS: a wave's keys and values come out of LDS at the
// rate at which the matrix units take them, and the softmax between the two
// products is what has to hide behind the other wave of the SIMD.  While a
// tile is multiplied another is on its way to LDS (an 8-bit cache through
// registers): the next, or with eight waves the one after it, so that a tile
// has landed a tile before it is used.  One barrier a tile.
//
// Many row tiles keep the GPU busy by themselves, the longest started first.
// Few of them (a short chunk behind a long cache, one KV head) are cut along
// the keys, like decode's requests: equal shares of the work, one for each
// workgroup that fits the GPU at once, and a second kernel that joins the row
// tiles that were cut.
#include <type_traits>

#include "attention_internal.h"
#include "attention_mfma.h"

namespace topkv_attend {

namespace {

constexpr int kTile = 64;                // keys
constexpr int kWaveRows = 32;
constexpr int kFew = 4, kMany = 8;       // waves of a workgroup
// The maximum that scores are taken relative to follows only when it is this far behind (in powers of two): weights
// stay below 2^8, which either 16-bit type holds as exactly as those below 1, and most tiles need no rescaling.
constexpr float kSlack = 8.f;
// Below this reference a weight's exponent may be made in one fused step, half a unit in its product's last place off.
// Making them all in two takes 1225 us instead of 1192 (8192 tokens, heads of 128).
constexpr float kFar = 1 << 18;

constexpr int resident(int KD) { return KD <= 64 ? 768 : KD <= 128 ? 512 : 256; }   // workgroups of 4 waves that 256 CUs hold
constexpr int kLeast = 4;                // key tiles of a share, at least
constexpr int kCutRows = kFew * kWaveRows;

struct Plan {
  int32_t most;        // row tiles that ascending q_starts can make
  int32_t shares;      // wanted; 0: a workgroup per row tile
  float* part;         // [2 * share + 1 for a row tile's first piece][kv head][kCutRows][head_dim]
  float2v* part_ml;    // the same without head_dim: maximum and sum
  int4* cut;           // [share]: request and first row of the row tile that starts in it and goes on, pieces (0: none)
};

struct Rows {          // one request's new tokens
  int32_t first, count, shift;           // in q; shift: position of the first of them

  template <int kRows> __device__ int32_t tiles(const Args& a) const {
    return (int32_t)(((int64_t)count * a.group + kRows - 1) / kRows);
  }
  // what the rows of row tile i see
  template <int kRows> __device__ Span span(const Args& a, int32_t i) const {
    const int64_t rows = (int64_t)count * a.group, last = (int64_t)(i + 1) * kRows < rows ? (int64_t)(i + 1) * kRows : rows;
    return key_span(a, shift + token_of(a, i * kRows), shift + token_of(a, (int32_t)last - 1));
  }
  // key tiles of the last row tile, at least 1: every row tile of the request counts as this many when work is shared out
  template <int kRows> __device__ int32_t depth(const Args& a) const {
    const int32_t n = (span<kRows>(a, tiles<kRows>(a) - 1).count + kTile - 1) / kTile;
    return n < 1 ? 1 : n;
  }
};

__device__ __forceinline__ Rows rows_of(const Args& a, int32_t r) {
  Rows w;
  w.first = clamped_start(a, r);
  const int32_t end = clamped_start(a, r + 1);
  w.count = end > w.first ? end - w.first : 0;
  w.shift = clamped_len(a, r) - w.count;
  return w;
}

// Eight 16-bit values with infinities and NaN as zeros; *any is set where there were some.
template <int T>
__device__ __forceinline__ uint4v without_special(uint4v w, bool* any) {
  constexpr uint32_t e = T == TOPKV_BF16 ? 0x7f80u : 0x7c00u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool lo = (w[i] & e) == e, hi = (w[i] >> 16 & e) == e;
    *any |= lo | hi;
    w[i] &= (lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u);
  }
  return w;
}

constexpr int kAhead = 2;                // steps of the first product that keys are read ahead

// Whether cutting row tiles along the keys takes less time than leaving them whole, both estimated in key tiles of a
// workgroup alone on its CU (1.8 us; two on a CU take 1.4 as long each).  Whole: the deepest row tile, or the work of
// all over the workgroups that fit.  Cut: an equal share, and for shorter prologues, partial results and the join 8 and
// up to 12 more, by how many pieces there are.  One request, 8 KV heads of 4, 3000 new tokens: whole 100 us, cut 217;
// 64 new tokens of 3000: 92 and 37.
template <int kWaves, int KD>
__device__ bool pays(const Args& a) {
  constexpr int kRows = kWaveRows * kWaves;
  __shared__ float s_units[kWaves], s_work[kWaves], s_deep[kWaves], s_tiles[kWaves];
  float units = 0.f, work = 0.f, deep = 0.f, tiles = 0.f;
  for (int32_t r = threadIdx.x; r < a.num_reqs; r += 64 * kWaves) {
    const Rows w = rows_of(a, r);
    const int32_t n = w.tiles<kRows>(a);
    if (n == 0) continue;
    const float d = (float)w.depth<kRows>(a), first = (float)((w.span<kRows>(a, 0).count + kTile - 1) / kTile);
    tiles += n;
    units += n * d;
    work += n * 0.5f * (first + d);
    deep = fmaxf(deep, d);
  }
#pragma unroll
  for (int i = 32; i; i >>= 1) {
    units += __shfl_xor(units, i, 64);
    work += __shfl_xor(work, i, 64);
    tiles += __shfl_xor(tiles, i, 64);
    deep = fmaxf(deep, __shfl_xor(deep, i, 64));
  }
  if ((threadIdx.x & 63) == 0) {
    const int w = threadIdx.x >> 6;
    s_units[w] = units, s_work[w] = work, s_deep[w] = deep, s_tiles[w] = tiles;
  }
  __syncthreads();
  units = work = deep = tiles = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    units += s_units[w], work += s_work[w], tiles += s_tiles[w];
    deep = fmaxf(deep, s_deep[w]);
  }
  const float fit = (float)resident(KD), heads = (float)a.kv_heads, slow = tiles * heads <= 256.f ? 1.f : 1.4f;
  const float share = units * heads / fit, whole = fmaxf(deep, work * heads / fit) * slow;
  const float cut = fmaxf(share, (float)kLeast) * 1.4f + 8.f + 12.f * fminf(1.f, share / kLeast);
  return cut < whole;
}

template <int T, bool kF8, int KD, int kWaves, bool kCut>
__global__ __launch_bounds__(64 * kWaves, resident(KD) / 256) void kv_attention_prompt_kernel(Args a, Plan plan) {
  typedef typename Elem<T>::vec8 vec8;
  typedef typename Elem<T>::type elem;
  constexpr int kThreads = 64 * kWaves, kRows = kWaveRows * kWaves;
  constexpr int NC = KD / 8;                                     // 16-byte chunks of a row in LDS
  constexpr int kLoads = kTile * NC / kThreads;                  // of a thread, for the keys and again for the values
  constexpr int kHalf = kTile * KD * 2;                          // bytes of a tile's keys
  constexpr int kBuffers = kWaves == kMany && !kF8 ? 3 : 2;      // tiles in LDS: one in use, the others on their way
  __shared__ __attribute__((aligned(16))) char s_tile[kBuffers][2 * kHalf];
  __shared__ int32_t s_special[kBuffers][kWaves];
  __shared__ int32_t s_request;
  __shared__ int64_t s_base;
  __shared__ Rows s_rows;

  const int wave = threadIdx.x >> 6;

  // KV heads side by side: with 8 of them an XCD sees the keys and values of one, which its L2 then serves to all row
  // tiles (8192 tokens, 8 heads of 128: 1204 us, against 1257 with all heads on every XCD).
  const int32_t number = blockIdx.x / a.kv_heads, kv_head = blockIdx.x - number * a.kv_heads;
  bool cutting = false;                                          // whether this batch is cut: the same for all workgroups
  if constexpr (kCut) {
    if (number < plan.shares && kv_head == 0 && threadIdx.x == 0) plan.cut[number] = make_int4(0, 0, 0, 0);
    cutting = pays<kWaves, KD>(a);
    if (cutting && number >= plan.shares) return;
  }
  Rows mine;
  const auto weight = [&](int32_t r) -> int64_t {
    mine = rows_of(a, r);
    const int32_t n = mine.tiles<kRows>(a);
    return cutting && n > 0 ? (int64_t)n * mine.depth<kRows>(a) : n;
  };
  if (threadIdx.x == 0) s_request = -1;
  Scan<int64_t> scan = scan_requests<int64_t, kWaves>(a.num_reqs, weight);
  int64_t size = 1, at, upto;
  if (cutting) {
    size = (scan.total + plan.shares - 1) / plan.shares;
    size = size < kLeast ? kLeast : size;
    at = number * size;
    upto = at + size < scan.total ? at + size : scan.total;
  } else {
    if (scan.total > plan.most) return;                          // q_starts do not ascend
    at = scan.total - 1 - number;                                // the last, longest first
    upto = at + 1;
  }
  if (at >= 0 && scan.holds(at)) {
    s_request = scan.lo + 1 < scan.hi ? scan.find(at, weight) : scan.lo;   // the thread's only request is still in hand
    s_base = scan.base;
    s_rows = mine;
  }
  __syncthreads();
  int32_t request = __builtin_amdgcn_readfirstlane(s_request);
  if (request < 0) return;
  int64_t base = s_base;
  mine = s_rows;

  const char* cache = a.cache + (int64_t)kv_head * a.head_bytes;
  const int32_t chunks = a.head_dim / 8;
  constexpr int kChunkBytes = kF8 ? 8 : 16;
  typedef typename std::conditional<kF8, uint2v, uint4v>::type Raw;
  if (chunks < NC) {                                             // padding stays zero: loads leave it alone
    for (int i = threadIdx.x; i < kBuffers * 2 * kHalf / 16; i += kThreads)
      *reinterpret_cast<uint4v*>(&s_tile[0][0] + i * 16) = uint4v{0, 0, 0, 0};
    __syncthreads();
  }

  while (at < upto) {
  int lane = threadIdx.x & 63;
  if constexpr (kCut) asm volatile("" : "+v"(lane));             // addresses made from it stay in the loop: registers
  const int col = lane & 31, half = lane >> 5;
  int32_t row_tile = (int32_t)(at - base);
  int32_t key_from = 0, key_to = INT32_MAX;                      // key tiles of this piece
  bool whole = true, opens = true;
  if (cutting) {
    const int32_t depth = mine.depth<kRows>(a);
    row_tile = (int32_t)((at - base) / depth);
    const int32_t from = (int32_t)((at - base) - (int64_t)row_tile * depth);
    const int32_t to = upto - at < depth - from ? from + (int32_t)(upto - at) : depth;
    const int32_t have = (mine.span<kRows>(a, row_tile).count + kTile - 1) / kTile;
    key_from = (int32_t)((int64_t)have * from / depth);
    key_to = (int32_t)((int64_t)have * to / depth);
    opens = from == 0;
    whole = opens && to == depth;
    if (opens && !whole && kv_head == 0 && threadIdx.x == 0)
      plan.cut[number] = make_int4(request, row_tile * kRows, (int32_t)((at + depth - 1) / size) - number + 1, 0);
    at += to - from;
  } else {
    at = upto;
  }
  const int32_t first_row = row_tile * kRows;
  const int32_t q_first = mine.first, shift = mine.shift;
  const int64_t rows = (int64_t)mine.count * a.group;
  const int32_t last_row = (int32_t)(first_row + kRows < rows ? first_row + kRows : rows) - 1;
  const Span span = mine.span<kRows>(a, row_tile);

  // this lane's row, and the positions of the wave's rows
  const int32_t row = first_row + wave * kWaveRows + col;
  const bool real = row < rows;
  const int32_t token = token_of(a, row), pos = real ? shift + token : -1;
  const int32_t head = kv_head * a.group + (row - token * a.group);
  const int32_t wave_row = first_row + wave * kWaveRows;
  const int32_t wave_first = shift + token_of(a, wave_row);
  const int32_t wave_last =
      wave_row < rows ? shift + token_of(a, (int32_t)(wave_row + kWaveRows < rows ? wave_row + kWaveRows - 1 : rows - 1)) : -1;

  vec8 q[KD / 16];
  {
    const char* from = static_cast<const char*>(a.q) + ((int64_t)(q_first + token) * a.q_stride + (int64_t)head * a.head_dim) * 2;
#pragma unroll
    for (int s = 0; s < KD / 16; ++s) {
      const int d = s * 16 + half * 8;
      union {
        uint4v w;
        vec8 v;
      } u;
      u.w = uint4v{0, 0, 0, 0};
      if (real && d < a.head_dim) u.w = *reinterpret_cast<const uint4v*>(from + 2 * d);
      q[s] = u.v;
    }
  }

  const int32_t* table = a.tables + (int64_t)request * a.bt_stride;
  float16v acc[KD / 32];
#pragma unroll
  for (int t = 0; t < KD / 32; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[t][i] = 0.f;
  float m = -INFINITY, l = 0.f;
  float slack = kSlack;

  // Lane k of every wave looks after key k of the tile: its table entry is asked for before the tile's rows of the
  // step before, its row's offset is handed to the lanes that load the row.  Where rows go straight to LDS the compiler
  // does not see their loads, and waits for them too where it uses the entry.
  const auto ask = [&](int32_t first) -> int32_t {
    const int32_t v = first + lane;
    return v < span.count ? table[page_of(a, (uint32_t)key_position(span, v))] : -1;
  };
  const auto locate = [&](int32_t first, int32_t entry) -> int64_t {
    const int32_t v = first + lane;
    if (v >= span.count || entry < 0 || entry >= a.num_pages) return -1;
    const uint32_t j = (uint32_t)key_position(span, v);
    return (int64_t)entry * a.page_bytes + (int64_t)(j - page_of(a, j) * (uint32_t)a.page_size) * a.slot_bytes;
  };
  // The lane again, where addresses made from it had better be made anew in every tile than be kept.
  const auto near = [&]() -> int {
    int here = lane;
    if constexpr (kCut || KD > 128) asm volatile("" : "+v"(here));
    return here;
  };
  const auto from_of = [&](int64_t off, int r) {
    const int lo = off < 0 ? 0 : (int)(uint32_t)off, hi = off < 0 ? 0 : (int)(off >> 32);
    return cache + (int64_t)((uint64_t)(uint32_t)__shfl(hi, r, 64) << 32 | (uint32_t)__shfl(lo, r, 64));
  };
  // An 8-bit cache passes through registers, where it is widened; 16-bit rows go from memory straight to LDS, a place
  // 16 bytes behind the other by lane, so the swizzle is in which chunk a lane asks for.
  Raw rk[kF8 ? kLoads : 1], rv[kF8 ? kLoads : 1];
  const auto fetch = [&](int buf, int64_t off) {
    const int lane = near();
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int place = (wave * kLoads + i) * 64 + lane, r = place / NC, c = (place - r * NC) ^ swizzle<NC>(r);
      const char* from = from_of(off, r) + c * kChunkBytes;
      if constexpr (kF8) {
        if (c < chunks) {
          rk[i] = *reinterpret_cast<const Raw*>(from);
          rv[i] = *reinterpret_cast<const Raw*>(from + a.value_bytes);
        }
      } else if (c < chunks) {
        load_to_lds(s_tile[buf] + (wave * kLoads + i) * 1024, from);
        load_to_lds(s_tile[buf] + kHalf + (wave * kLoads + i) * 1024, from + a.value_bytes);
      }
    }
  };
  // The tile is in LDS for this wave's rows: rows without a key as zeros, whatever their place holds, and (watch) its
  // values' infinities and NaN as zeros too: times a weight of 0 they would reach rows that do not see their token.
  // Rows that do see it get them afterwards.
  const auto settle = [&](int buf, uint64_t there, bool watch, bool more) {
    if constexpr (!kF8) {
      // more: the loads of the tile after it are under way too (all of them: narrower rows may have a load without a
      // lane to it, which is never issued)
      if (kBuffers == 3 && more && chunks == NC) asm volatile("s_waitcnt vmcnt(%0)" ::"i"(2 * kLoads) : "memory");
      else wait_loads();
      if (there == ~0ull && !watch) return;
    }
    bool special = false;
    const int lane = near();
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int place = (wave * kLoads + i) * 64 + lane, r = place / NC, c = (place - r * NC) ^ swizzle<NC>(r);
      uint4v* k = reinterpret_cast<uint4v*>(s_tile[buf] + place * 16);
      uint4v* v = reinterpret_cast<uint4v*>(s_tile[buf] + kHalf + place * 16);
      if (c < chunks) {
        const bool is = there >> r & 1;
        const uint4v none = {0, 0, 0, 0};
        if constexpr (kF8) {
          *k = is ? widen<T>(rk[i]) : none;
          const uint4v w = widen<T>(rv[i]);
          *v = !is ? none : watch ? without_special<T>(w, &special) : w;
        } else {
          if (!is) *k = *v = none;
          else if (watch) *v = without_special<T>(*v, &special);
        }
      }
    }
    const bool any = __any(special);
    if (lane == 0) s_special[buf][wave] = any;
  };
  // Whether every key of the tile is seen by every row with positions [p0, p1] (a tile across the seam between the
  // first tokens and the window is never taken for such).
  const auto open = [&](int32_t first, int32_t p0, int32_t p1) -> bool {
    if (first + kTile > span.count || p0 < 0) return false;
    const int32_t k0 = key_position(span, first), k1 = key_position(span, first + kTile - 1);
    return (k1 <= p0) & ((a.window == 0) | (k0 > p1 - a.window) | (k1 < a.sinks));
  };

  const int32_t count = (int64_t)key_to * kTile < span.count ? key_to * kTile : span.count;   // end of the piece's keys
  const int32_t begin = key_from * kTile;
  const int32_t wg_first = shift + token_of(a, first_row), wg_last = shift + token_of(a, last_row);
  int64_t off = locate(begin, ask(begin));
  int32_t entry = ask(begin + kTile);
  uint64_t there = __ballot(off >= 0), there1 = 0, there2 = 0;   // which keys the tile, the next and the one after it have
  if (begin < count) fetch(0, off);
  if constexpr (kBuffers == 3) {
    off = locate(begin + kTile, entry);
    entry = ask(begin + 2 * kTile);
    there1 = __ballot(off >= 0);
    if (begin + kTile < count) fetch(1, off);
  }
  // Whether not all rows of the workgroup see the whole tile: then its values were looked over, for the rows of every wave.
  bool watch = !open(begin, wg_first, wg_last);
  if (begin < count) settle(0, there, watch, begin + kTile < count);
  if constexpr (kF8) {
    if (begin + kTile < count) {
      off = locate(begin + kTile, entry);
      entry = ask(begin + 2 * kTile);
      there1 = __ballot(off >= 0);
      fetch(1, off);
    }
  }
  __syncthreads();

  int buf = 0;
  for (int32_t first = begin; first < count; first += kTile) {
    const int next = buf + 1 < kBuffers ? buf + 1 : 0;
    const char* keys = s_tile[buf];
    const char* values = keys + kHalf;
    if constexpr (!kF8) {
      constexpr int kOn = (kBuffers - 1) * kTile;
      if (first + kOn < count) {
        off = locate(first + kOn, entry);
        entry = ask(first + kOn + kTile);
        (kBuffers == 3 ? there2 : there1) = __ballot(off >= 0);
        fetch(kBuffers == 2 ? next : next + 1 < kBuffers ? next + 1 : 0, off);
      }
    }
    // tiles behind the wave's last row, or (their last key) before its first row's window, are nothing to it
    const int32_t k_first = key_position(span, first);
    const int32_t k_last = key_position(span, first + kTile - 1 < count ? first + kTile - 1 : count - 1);
    const bool use = k_first <= wave_last && (a.window == 0 || k_last > wave_first - a.window || k_first < a.sinks);
    if (use) {
      // Keys leave LDS a few steps ahead of their product, values and weights one step ahead of theirs: the scheduling
      // barriers hold that order, which the compiler gives up for fewer registers (a product then waits for LDS each time).
      float16v x[2];
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) x[b][i] = 0.f;
      const int lane = near(), col = lane & 31, half = lane >> 5;
      const auto key = [&](int b, int s) {
        const int r = b * 32 + col;
        return *reinterpret_cast<const vec8*>(keys + (r * NC + ((s * 2 + half) ^ swizzle<NC>(r))) * 16);
      };
      constexpr int kSteps = KD / 16;
      vec8 k[kAhead + 1][2];
#pragma unroll
      for (int s = 0; s < kAhead; ++s)
#pragma unroll
        for (int b = 0; b < 2; ++b) k[s][b] = key(b, s);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        if (s + kAhead < kSteps)
#pragma unroll
          for (int b = 0; b < 2; ++b) k[(s + kAhead) % (kAhead + 1)][b] = key(b, s + kAhead);
#pragma unroll
        for (int b = 0; b < 2; ++b) x[b] = Elem<T>::mfma32(k[s % (kAhead + 1)][b], q[s], x[b]);
        __builtin_amdgcn_sched_barrier(0);
      }
      const bool clear = there == ~0ull && open(first, wave_first, wave_last);
      if (!clear) {
        if (there != ~0ull) {
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            const uint32_t is = (uint32_t)(there >> (b * 32)) >> (half * 4);
#pragma unroll
            for (int i = 0; i < 16; ++i) x[b][i] = is >> ((i >> 2) * 8 + (i & 3)) & 1 ? x[b][i] : -INFINITY;
          }
        }
        // The row sees key numbers below `few` (first tokens) and `wide` ones from `from` on, here counted from the lane's
        // first key of the tile: two comparisons a key.
        const int32_t here = first + half * 4, behind = span.head - span.start;
        const int32_t last = pos + behind, from = (a.window > 0 ? last - a.window + 1 : 0) - here;
        const int32_t few = (a.sinks + behind < last + 1 ? a.sinks + behind : last + 1) > span.head
                                ? (a.sinks + behind < last + 1 ? a.sinks + behind : last + 1) - here
                                : span.head - here;
        const uint32_t wide = pos < 0 ? 0u : (uint32_t)(last + 1 - here - from);
        const int32_t firsts = pos < 0 ? INT32_MIN : few;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int32_t k = b * 32 + (i >> 2) * 8 + (i & 3);
            const bool seen = (k < firsts) | ((uint32_t)(k - from) < wide);
            x[b][i] = seen ? x[b][i] : -INFINITY;
          }
      }
      float top = -INFINITY;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, x[b][i]);
      top = reference<T>(max_halves(top), a.scale, kSlack);
      float base = m == -INFINITY ? 0.f : m, scale = a.scale;
      if (__builtin_expect(__any(top - m > slack), 0)) {         // some row's scores left the maximum behind
        const float up = fmaxf(m, top), fall = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - up);
        m = up;
        l *= fall;
#pragma unroll
        for (int t = 0; t < KD / 32; ++t) acc[t] *= fall;
        base = m == -INFINITY ? 0.f : m;
        if (__any(__builtin_fabsf(base) > kFar)) {
          slack = -INFINITY;                                     // and so in every tile from here on
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) x[b][i] = exponent_of(x[b][i], scale, base);
          base = 0.f;
          scale = 1.f;
        }
      }
      // weights of 16 keys
      const auto weigh = [&](int s) {
        vec8 p;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float w = __builtin_amdgcn_exp2f(fmaf(x[s >> 1][(s & 1) * 8 + i], scale, -base));
          l += w;
          p[i] = (elem)w;                                        // rounded for the matrix units, its sum is not
        }
        return p;
      };
      // values by columns: lane (d, half) takes keys 4 half .. + 3 of each eight, as the weights lie
      const auto column = [&](int t, int s) {
        union {
          uint2v h[2];
          vec8 v;
        } u;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int r = s * 16 + e * 8 + half * 4 + (lane >> 2 & 3), c = t * 4 + (lane >> 4 & 1) * 2 + (lane >> 1 & 1);
          u.h[e] = read_transposed(values + (r * NC + (c ^ swizzle<NC>(r))) * 16 + (lane & 1) * 8);
        }
        return u.v;
      };
      constexpr int kWide = KD == 128 ? 4 : 2;                   // 32-element columns of a step
      constexpr int kTurns = KD / 32 / kWide;                    // steps of the same 16 keys
      vec8 v[2][kWide], p[2];
#pragma unroll
      for (int t = 0; t < kWide; ++t) v[0][t] = column(t, 0);
      p[0] = weigh(0);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int n = 0; n < 4 * kTurns; ++n) {
        const int s = n / kTurns, u = n % kTurns;
        if (n + 1 < 4 * kTurns)
#pragma unroll
          for (int t = 0; t < kWide; ++t) v[(n + 1) & 1][t] = column((n + 1) % kTurns * kWide + t, (n + 1) / kTurns);
#pragma unroll
        for (int t = 0; t < kWide; ++t) acc[u * kWide + t] = Elem<T>::mfma32(v[n & 1][t], p[s & 1], acc[u * kWide + t]);
        if (u == 0 && s + 1 < 4) p[(s + 1) & 1] = weigh(s + 1);
        __builtin_amdgcn_sched_barrier(0);
      }
      // `watch` alone would do (a wave that is not clear has none but looked-over tiles, or a word that says so), but the
      // branch that such a wave takes anyway keeps registers free: 8192 tokens 1196 us and 1218, windows 161 and 175.
      if (!clear || watch) {
        int special = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) special |= s_special[buf][w];
        if (special) {
          const int64_t at = locate(first, ask(first));
          const int32_t low = a.window > 0 ? pos - a.window : -1;
#pragma unroll 1
          for (int k = 0; k < kTile && first + k < count; ++k) {
            const int32_t j = key_position(span, first + k);
            const bool seen = (there >> k & 1) & (j <= pos) & ((j > low) | (j < a.sinks));
            const char* v = from_of(at, k) + a.value_bytes + half * 4 * (kF8 ? 1 : 2);
#pragma unroll
            for (int t = 0; t < KD / 32; ++t)
#pragma unroll
              for (int o = 0; o < 4; ++o)
                if (t * 32 + o * 8 < a.head_dim)                 // the same in all lanes
#pragma unroll
                  for (int i = 0; i < 4; ++i) {
                    const float f = Load<kF8 ? TOPKV_FP8_E4M3 : T>::at(v + (t * 32 + o * 8 + i) * (kF8 ? 1 : 2));
                    acc[t][o * 4 + i] += (seen & !(__builtin_fabsf(f) < INFINITY)) ? f : 0.f;
                  }
          }
        }
      }
    }
    watch = !open(first + kTile, wg_first, wg_last);
    if (first + kTile < count) settle(next, there1, watch, first + 2 * kTile < count);
    there = there1;
    if constexpr (kBuffers == 3) there1 = there2;
    if constexpr (kF8) {
      if (first + 2 * kTile < count) {
        off = locate(first + 2 * kTile, entry);
        entry = ask(first + 3 * kTile);
        there1 = __ballot(off >= 0);
        fetch(buf, off);
      }
    }
    buf = next;
    __syncthreads();
  }

  l = sum_halves(l);
  if (!whole) {
    if (real) {
      const int64_t slot = ((2 * (int64_t)number + opens) * a.kv_heads + kv_head) * kRows + (row - first_row);
      float* out = plan.part + slot * a.head_dim;
#pragma unroll
      for (int t = 0; t < KD / 32; ++t)
#pragma unroll
        for (int o = 0; o < 4; ++o)
          if (t * 32 + o * 8 < a.head_dim)
            *reinterpret_cast<float4v*>(out + t * 32 + o * 8 + half * 4) =
                float4v{acc[t][o * 4], acc[t][o * 4 + 1], acc[t][o * 4 + 2], acc[t][o * 4 + 3]};
      if (half == 0) plan.part_ml[slot] = float2v{m, l};
    }
  } else {
    const float inv = l == 0.f ? 0.f : a.v_scale / l;
    elem* out = static_cast<elem*>(a.out) + (int64_t)(q_first + token) * a.out_stride + (int64_t)head * a.value_dim;
#pragma unroll
    for (int t = 0; t < KD / 32; ++t)
#pragma unroll
      for (int o = 0; o < 4; o += 2) {
        // 4 elements of chunk o and 4 of o + 1 a lane, the other 4 of each in the other half: exchanged, a lane has 8 of one
        union {
          elem e[8];
          uint4v w;
        } u;
#pragma unroll
        for (int i = 0; i < 8; ++i) u.e[i] = (elem)(l == 0.f ? 0.f : acc[t][o * 4 + i] * inv);
        const auto x = __builtin_amdgcn_permlane32_swap(u.w[0], u.w[2], false, false);
        const auto y = __builtin_amdgcn_permlane32_swap(u.w[1], u.w[3], false, false);
        u.w = uint4v{x[0], y[0], x[1], y[1]};
        const int d = t * 32 + (o + half) * 8;
        if (real && d < a.head_dim) {
          if (a.out_wide) {
            *reinterpret_cast<uint4v*>(out + d) = u.w;
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) out[d + i] = u.e[i];
          }
        }
      }
    if (real && a.lse && half == 0)
      a.lse[(int64_t)(q_first + token) * a.num_heads + head] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
  }
  if (cutting) {
    // on to the next row tile, of a later request where this one's are done
    if (at < upto && at == base + (int64_t)mine.tiles<kRows>(a) * mine.depth<kRows>(a)) {
      base = at;
      do mine = rows_of(a, ++request);
      while (mine.count == 0 && request + 1 < a.num_reqs);
    }
  }
  }
}

// Row tiles in pieces: a workgroup for 16 rows of (share that one starts in,
// KV head), 16 lanes a row with 8 elements each, so that every load of a wave
// is whole lines and no row waits for another.
template <int T>
__global__ __launch_bounds__(256) void kv_attention_prompt_join_kernel(Args a, Plan plan) {
  typedef typename Elem<T>::type elem;
  const int32_t share = blockIdx.x / a.kv_heads, kv_head = blockIdx.x - share * a.kv_heads;
  const int4 cut = plan.cut[share];
  if (cut.z == 0) return;
  const Rows mine = rows_of(a, cut.x);
  const int32_t in_tile = blockIdx.y * 16 + (threadIdx.x >> 4), row = cut.y + in_tile;
  if (row >= (int64_t)mine.count * a.group) return;
  const int32_t token = token_of(a, row), head = kv_head * a.group + (row - token * a.group);
  const int64_t step = (int64_t)a.kv_heads * kCutRows;
  const int64_t slot = (2 * (int64_t)share * a.kv_heads + kv_head) * kCutRows + in_tile;   // piece k: 2 k steps on, the first 1
  float top = -INFINITY;
#pragma unroll 4
  for (int32_t k = 0; k < cut.z; ++k) top = fmaxf(top, plan.part_ml[slot + (k ? 2 * k : 1) * step][0]);
  const float base = top == -INFINITY ? 0.f : top;
  float sum = 0.f;
  elem* out = static_cast<elem*>(a.out) + (int64_t)(mine.first + token) * a.out_stride + (int64_t)head * a.value_dim;
  for (int32_t d = (threadIdx.x & 15) * 8; d < a.head_dim; d += 128) {
    float4v lo = {0.f, 0.f, 0.f, 0.f}, hi = lo;
    sum = 0.f;
#pragma unroll 4
    for (int32_t k = 0; k < cut.z; ++k) {
      const int64_t s = slot + (k ? 2 * k : 1) * step;
      const float2v ml = plan.part_ml[s];
      const float f = __builtin_amdgcn_exp2f(ml[0] - base);
      const float4v* from = reinterpret_cast<const float4v*>(plan.part + s * a.head_dim + d);
      sum = fmaf(f, ml[1], sum);
      lo += from[0] * f;
      hi += from[1] * f;
    }
    const float inv = sum == 0.f ? 0.f : a.v_scale / sum;
    union {
      elem e[8];
      uint4v w;
    } u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      u.e[i] = (elem)(sum == 0.f ? 0.f : lo[i] * inv);
      u.e[i + 4] = (elem)(sum == 0.f ? 0.f : hi[i] * inv);
    }
    if (a.out_wide) {
      *reinterpret_cast<uint4v*>(out + d) = u.w;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) out[d + i] = u.e[i];
    }
  }
  if (a.lse && (threadIdx.x & 15) == 0)
    a.lse[(int64_t)(mine.first + token) * a.num_heads + head] =
        sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

// Row tiles that any division of the rows among the requests can make, and that every one makes.
int64_t most_tiles(const Args& a, int waves) { return (int64_t)a.total_q * a.group / (waves * kWaveRows) + a.num_reqs; }
int64_t least_tiles(const Args& a, int waves) {
  return ((int64_t)a.total_q * a.group + waves * kWaveRows - 1) / (waves * kWaveRows);
}

int64_t most_keys(const Args& a) {
  const int64_t seen = (int64_t)a.bt_stride * a.page_size;
  return a.window > 0 && (int64_t)a.window + a.sinks < seen ? (int64_t)a.window + a.sinks : seen;
}

// Eight waves on one tile halve the loads of a row and ask for it a tile earlier, four waves twice over a CU start and
// end more easily.  8192 tokens, heads of 128: 8 waves 1204 us, 4 1278; windows of 128, heads of 64, in
// an earlier form: 250 and 180.  Heads of 256 have no registers for more than one wave a SIMD.
int waves_for(const Args& a) {
  return a.head_dim > 64 && a.head_dim <= 128 && most_keys(a) >= 1024 &&
                 least_tiles(a, kMany) * a.kv_heads >= resident(a.head_dim)
             ? kMany
             : kFew;
}

// Shares of the work where it may be cut, which the kernel decides by the lengths; 0 where the row tiles are enough for
// certain (twice as many as fit the GPU at once) or no row can see more keys than two shares should have.
int32_t most_shares(const Args& a) {
  const int32_t n = resident(a.head_dim) / a.kv_heads;
  return most_keys(a) <= 2 * kLeast * kTile ? 0 : n < 1 ? 1 : n;
}
int32_t wanted_shares(const Args& a) {
  return least_tiles(a, kFew) * a.kv_heads >= 2 * resident(a.head_dim) ? 0 : most_shares(a);
}

int64_t up16(int64_t x) { return (x + 15) / 16 * 16; }

template <int T, bool kF8, int KD, int kWaves, bool kCut>
void launch_one(const Args& a, const Plan& p, int64_t items, hipStream_t stream) {
  hipLaunchKernelGGL(HIP_KERNEL_NAME(kv_attention_prompt_kernel<T, kF8, KD, kWaves, kCut>), dim3((unsigned)(items * a.kv_heads)),
                     dim3(64 * kWaves), 0, stream, a, p);
}

template <int T, bool kF8>
void launch(const Args& a, const Plan& p, hipStream_t stream) {
  if (p.shares > 0) {
    const int64_t items = p.most > p.shares ? p.most : p.shares;   // the kernel finds out which of them are wanted
    if (a.head_dim <= 64) launch_one<T, kF8, 64, kFew, true>(a, p, items, stream);
    else if (a.head_dim <= 128) launch_one<T, kF8, 128, kFew, true>(a, p, items, stream);
    else launch_one<T, kF8, 256, kFew, true>(a, p, items, stream);
    hipLaunchKernelGGL(HIP_KERNEL_NAME(kv_attention_prompt_join_kernel<T>), dim3((unsigned)(p.shares * a.kv_heads), kCutRows / 16),
                       dim3(256), 0, stream, a, p);
  } else if (a.head_dim <= 64) {
    launch_one<T, kF8, 64, kFew, false>(a, p, p.most, stream);
  } else if (waves_for(a) == kMany) {
    launch_one<T, kF8, 128, kMany, false>(a, p, p.most, stream);
  } else if (a.head_dim <= 128) {
    launch_one<T, kF8, 128, kFew, false>(a, p, p.most, stream);
  } else {
    launch_one<T, kF8, 256, kFew, false>(a, p, p.most, stream);
  }
}

}  // namespace

bool prompt_geometry(const Args& a) {
  const int64_t unit = a.kv_dtype == TOPKV_FP8_E4M3 ? 8 : 16;
  return a.value_bytes != 0 && a.head_dim % 8 == 0 && a.head_dim <= 256 && a.slot_bytes % unit == 0 &&
         a.head_bytes % unit == 0 && a.page_bytes % unit == 0 && a.value_bytes % unit == 0 &&
         (int64_t)most_shares(a) * a.kv_heads <= kMostGroups;
}

bool prompt_takes(const Args& a) { return prompt_geometry(a) && most_tiles(a, kFew) * a.kv_heads <= kMostGroups; }

// For any number of tokens: fewer may be cut where more are not.
int64_t prompt_workspace(const Args& a) {
  if (!prompt_geometry(a)) return 0;
  const int64_t shares = most_shares(a), rows = 2 * shares * a.kv_heads * kCutRows;
  return up16(rows * a.head_dim * 4) + up16(rows * 8) + shares * 16;
}

topkv_status_t run_prompt(const Args& a, void* workspace, hipStream_t stream) {
  Plan p = {};
  p.shares = wanted_shares(a);
  p.most = (int32_t)most_tiles(a, p.shares > 0 ? kFew : waves_for(a));
  if (p.shares > 0) {
    const int64_t rows = 2 * (int64_t)p.shares * a.kv_heads * kCutRows;
    char* at = static_cast<char*>(workspace);
    p.part = reinterpret_cast<float*>(at);
    at += up16(rows * a.head_dim * 4);
    p.part_ml = reinterpret_cast<float2v*>(at);
    at += up16(rows * 8);
    p.cut = reinterpret_cast<int4*>(at);
  }
  if (a.kv_dtype == TOPKV_FP8_E4M3) {
    if (a.dtype == TOPKV_BF16) launch<TOPKV_BF16, true>(a, p, stream);
    else launch<TOPKV_FP16, true>(a, p, stream);
  } else if (a.dtype == TOPKV_BF16) {
    launch<TOPKV_BF16, false>(a, p, stream);
  } else {
    launch<TOPKV_FP16, false>(a, p, stream);
  }
  return hipGetLastError() == hipSuccess ? TOPKV_OK : TOPKV_ERR_LAUNCH;
}

}  // namespace topkv_attend
