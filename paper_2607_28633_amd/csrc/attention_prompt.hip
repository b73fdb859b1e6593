// attention_prompt.hip - many new tokens per request on the matrix units.
//
// A workgroup takes 128 query rows of one KV head, a row being one (token,
// query head of the group): neighbouring tokens and all heads of the group
// read the same keys, so even a short chunk fills the rows.  Four waves of 32
// rows walk tiles of 64 keys: scores^T = K Q^T, running maximum and sum,
// out^T += V^T P^T, 4 * 32 * 64 * head_dim flops a wave and tile against
// 256 * head_dim bytes of LDS: a wave's keys and values come out of LDS at the
// rate at which the matrix units take them, and the softmax between the two
// products is what has to hide behind the other wave of the SIMD.  While a
// tile is multiplied the next one is on its way to registers and goes into the
// other half of a double buffer: one barrier a tile.
#include <type_traits>

#include "attention_internal.h"
#include "attention_mfma.h"

namespace topkv_attend {

namespace {

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kTile = 64;                // keys
constexpr int kWaveRows = 32;
constexpr int kRows = kWaves * kWaveRows;
// The maximum that scores are taken relative to follows only when it is this far behind (in powers of two): weights
// stay below 2^8, which either 16-bit type holds as exactly as those below 1, and most tiles need no rescaling.
constexpr float kSlack = 8.f;

__device__ __forceinline__ int32_t row_tiles(const Args& a, int32_t r) {
  const int32_t s = clamped_start(a, r), e = clamped_start(a, r + 1);
  return e > s ? (int32_t)(((int64_t)(e - s) * a.group + kRows - 1) / kRows) : 0;
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

template <int T, bool kF8, int KD>
__global__ __launch_bounds__(kThreads, KD > 128 ? 1 : 2) void kv_attention_prompt_kernel(Args a) {
  typedef typename Elem<T>::vec8 vec8;
  typedef typename Elem<T>::type elem;
  constexpr int NC = KD / 8;                                     // 16-byte chunks of a row in LDS
  constexpr int kLoads = kTile * NC / kThreads;                  // of a thread, for the keys and again for the values
  constexpr int kHalf = kTile * KD * 2;                          // bytes of a tile's keys
  __shared__ __attribute__((aligned(16))) char s_tile[2][2 * kHalf];
  __shared__ int32_t s_special[2][kWaves];
  __shared__ int32_t s_request, s_base;

  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = lane & 31, half = lane >> 5;

  // Which rows: eight row tiles side by side over the eight XCDs, a tile's KV heads one after the other on one XCD
  // (whose L2 then sees whole rows of the cache, and neighbouring row tiles the same keys), the last, longest first.
  const auto tiles = [&](int32_t r) { return row_tiles(a, r); };
  Scan scan = scan_requests<kWaves>(a.num_reqs, tiles);
  const int32_t eight = blockIdx.x / (8 * a.kv_heads), within = blockIdx.x - eight * 8 * a.kv_heads;
  const int32_t item = scan.total - 1 - (eight * 8 + (within & 7)), kv_head = within >> 3;
  if (item < 0) return;
  if (item >= scan.base && item < scan.base + scan.mine) {
    s_request = scan.find(item, tiles);
    s_base = scan.base;
  }
  __syncthreads();
  const int32_t request = __builtin_amdgcn_readfirstlane(s_request);
  const int32_t first_row = (item - __builtin_amdgcn_readfirstlane(s_base)) * kRows;

  const int32_t q_first = clamped_start(a, request), q_count = clamped_start(a, request + 1) - q_first;
  const int64_t rows = (int64_t)q_count * a.group;
  const int32_t shift = clamped_len(a, request) - q_count;       // position of the request's first new token
  const int32_t last_row = (int32_t)(first_row + kRows < rows ? first_row + kRows : rows) - 1;
  const Span span = key_span(a, shift + first_row / a.group, shift + last_row / a.group);

  // this lane's row, and the positions of the wave's rows
  const int32_t row = first_row + wave * kWaveRows + col;
  const bool real = row < rows;
  const int32_t token = row / a.group, pos = real ? shift + token : -1;
  const int32_t head = kv_head * a.group + (row - token * a.group);
  const int32_t wave_row = first_row + wave * kWaveRows;
  const int32_t wave_first = shift + wave_row / a.group;
  const int32_t wave_last =
      wave_row < rows ? shift + (int32_t)(wave_row + kWaveRows < rows ? wave_row + kWaveRows - 1 : rows - 1) / a.group : -1;

  vec8 q[KD / 16];
  {
    const char* at = static_cast<const char*>(a.q) + ((int64_t)(q_first + token) * a.q_stride + (int64_t)head * a.head_dim) * 2;
#pragma unroll
    for (int s = 0; s < KD / 16; ++s) {
      const int d = s * 16 + half * 8;
      union {
        uint4v w;
        vec8 v;
      } u;
      u.w = uint4v{0, 0, 0, 0};
      if (real && d < a.head_dim) u.w = *reinterpret_cast<const uint4v*>(at + 2 * d);
      q[s] = u.v;
    }
  }

  const int32_t* table = a.tables + (int64_t)request * a.bt_stride;
  const char* cache = a.cache + (int64_t)kv_head * a.head_bytes;
  const int32_t chunks = a.head_dim / 8;
  constexpr int kChunkBytes = kF8 ? 8 : 16;
  typedef typename std::conditional<kF8, uint2v, uint4v>::type Raw;

  if (chunks < NC) {                                             // padding stays zero: loads leave it alone
    for (int i = threadIdx.x; i < 2 * 2 * kHalf / 16; i += kThreads)
      *reinterpret_cast<uint4v*>(&s_tile[0][0] + i * 16) = uint4v{0, 0, 0, 0};
    __syncthreads();
  }

  float16v acc[KD / 32];
#pragma unroll
  for (int t = 0; t < KD / 32; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[t][i] = 0.f;
  float m = -INFINITY, l = 0.f;

  // Lane k of every wave looks after key k of the tile: its table entry is asked for before the tile's rows of the
  // step before, its row's offset is handed to the lanes that load the row.
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
  const auto from_of = [&](int64_t off, int r) {
    const int lo = off < 0 ? 0 : (int)(uint32_t)off, hi = off < 0 ? 0 : (int)(off >> 32);
    return cache + (int64_t)((uint64_t)(uint32_t)__shfl(hi, r, 64) << 32 | (uint32_t)__shfl(lo, r, 64));
  };
  // An 8-bit cache passes through registers, where it is widened; 16-bit rows go from memory straight to LDS, a place
  // 16 bytes behind the other by lane, so the swizzle is in which chunk a lane asks for.
  Raw rk[kF8 ? kLoads : 1], rv[kF8 ? kLoads : 1];
  const auto fetch = [&](int buf, int64_t off) {
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
  const auto settle = [&](int buf, uint64_t there, bool watch) {
    if constexpr (!kF8) {
      wait_loads();
      if (there == ~0ull && !watch) return;
    }
    bool special = false;
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
          *v = is ? without_special<T>(widen<T>(rv[i]), &special) : none;
        } else {
          if (!is) *k = none;
          *v = is ? without_special<T>(*v, &special) : none;
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

  const int32_t count = span.count;
  const int32_t wg_first = shift + first_row / a.group, wg_last = shift + last_row / a.group;
  int64_t off = locate(0, ask(0));
  int32_t entry = ask(kTile);
  uint64_t there = __ballot(off >= 0), there_next = 0;
  fetch(0, off);
  settle(0, there, !open(0, wg_first, wg_last));
  if constexpr (kF8) {
    if (kTile < count) {
      off = locate(kTile, entry);
      entry = ask(2 * kTile);
      there_next = __ballot(off >= 0);
      fetch(1, off);
    }
  }
  __syncthreads();

  for (int32_t first = 0, buf = 0; first < count; first += kTile, buf ^= 1) {
    const char* keys = s_tile[buf];
    const char* values = keys + kHalf;
    if constexpr (!kF8) {
      if (first + kTile < count) {
        off = locate(first + kTile, entry);
        entry = ask(first + 2 * kTile);
        there_next = __ballot(off >= 0);
        fetch(buf ^ 1, off);
      }
    }
    // tiles behind the wave's last row, or (their last key) before its first row's window, are nothing to it
    const int32_t k_first = key_position(span, first);
    const int32_t k_last = key_position(span, first + kTile - 1 < count ? first + kTile - 1 : count - 1);
    const bool use = k_first <= wave_last && (a.window == 0 || k_last > wave_first - a.window || k_first < a.sinks);
    if (use) {
      float16v x[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
#pragma unroll
        for (int i = 0; i < 16; ++i) x[b][i] = 0.f;
        const int r = b * 32 + col;
#pragma unroll
        for (int s = 0; s < KD / 16; ++s) {
          const vec8 k = *reinterpret_cast<const vec8*>(keys + (r * NC + ((s * 2 + half) ^ swizzle<NC>(r))) * 16);
          x[b] = Elem<T>::mfma32(k, q[s], x[b]);
        }
      }
      const bool clear = there == ~0ull && open(first, wave_first, wave_last);
      if (!clear) {
        const int32_t low = a.window > 0 ? pos - a.window : -1, behind = span.start - span.head;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const uint32_t is = (uint32_t)(there >> (b * 32)) >> (half * 4);
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int32_t k = first + b * 32 + (i >> 2) * 8 + half * 4 + (i & 3);
            const int32_t j = k < span.head ? k : k + behind;
            const bool seen = (is >> ((i >> 2) * 8 + (i & 3)) & 1) & (j <= pos) & ((j > low) | (j < a.sinks));
            x[b][i] = seen ? x[b][i] : -INFINITY;
          }
        }
      }
      float top = -INFINITY;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, x[b][i]);
      top = max_halves(top) * a.scale;
      if (__any(top > m + kSlack)) {                             // some row's scores left the maximum behind
        const float up = fmaxf(m, top), fall = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - up);
        m = up;
        l *= fall;
#pragma unroll
        for (int t = 0; t < KD / 32; ++t) acc[t] *= fall;
      }
      const float base = m == -INFINITY ? 0.f : m;
      vec8 p[4];                                                 // 16 keys each
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float w = __builtin_amdgcn_exp2f(fmaf(x[b][i], a.scale, -base));
          l += w;
          p[b * 2 + (i >> 3)][i & 7] = (elem)w;                  // rounded for the matrix units, its sum is not
        }
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
#pragma unroll
      for (int t = 0; t < KD / 32; ++t)
#pragma unroll
        for (int s = 0; s < 4; ++s) acc[t] = Elem<T>::mfma32(column(t, s), p[s], acc[t]);
      if (!clear) {
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
                    acc[t][o * 4 + i] += seen & !(__builtin_fabsf(f) < INFINITY) ? f : 0.f;
                  }
          }
        }
      }
    }
    there = there_next;
    if (first + kTile < count) settle(buf ^ 1, there, !open(first + kTile, wg_first, wg_last));
    if constexpr (kF8) {
      if (first + 2 * kTile < count) {
        off = locate(first + 2 * kTile, entry);
        entry = ask(first + 3 * kTile);
        there_next = __ballot(off >= 0);
        fetch(buf, off);
      }
    }
    __syncthreads();
  }

  l = sum_halves(l);
  if (!real) return;
  const float inv = l == 0.f ? 0.f : a.v_scale / l;
  elem* out = static_cast<elem*>(a.out) + (int64_t)(q_first + token) * a.out_stride + (int64_t)head * a.value_dim;
#pragma unroll
  for (int t = 0; t < KD / 32; ++t)
#pragma unroll
    for (int o = 0; o < 4; ++o)
      if (t * 32 + o * 8 < a.head_dim)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          out[t * 32 + o * 8 + half * 4 + i] = (elem)(l == 0.f ? 0.f : acc[t][o * 4 + i] * inv);
  if (a.lse && half == 0)
    a.lse[(int64_t)(q_first + token) * a.num_heads + head] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

template <int T, bool kF8>
void launch(const Args& a, int64_t items, hipStream_t stream) {
  const dim3 grid((unsigned)((items + 7) / 8 * 8 * a.kv_heads)), block(kThreads);
  if (a.head_dim <= 64)
    hipLaunchKernelGGL(HIP_KERNEL_NAME(kv_attention_prompt_kernel<T, kF8, 64>), grid, block, 0, stream, a);
  else if (a.head_dim <= 128)
    hipLaunchKernelGGL(HIP_KERNEL_NAME(kv_attention_prompt_kernel<T, kF8, 128>), grid, block, 0, stream, a);
  else
    hipLaunchKernelGGL(HIP_KERNEL_NAME(kv_attention_prompt_kernel<T, kF8, 256>), grid, block, 0, stream, a);
}

// Row tiles that any division of the rows among the requests can make.
int64_t most_tiles(const Args& a) { return (int64_t)a.total_q * a.group / kRows + a.num_reqs; }

}  // namespace

bool prompt_takes(const Args& a) {
  const int64_t unit = a.kv_dtype == TOPKV_FP8_E4M3 ? 8 : 16;
  if (a.value_bytes == 0 || a.head_dim % 8 != 0 || a.head_dim > 256) return false;
  if (a.slot_bytes % unit != 0 || a.head_bytes % unit != 0 || a.page_bytes % unit != 0 || a.value_bytes % unit != 0) return false;
  return (most_tiles(a) + 8) * a.kv_heads <= INT32_MAX;
}

topkv_status_t run_prompt(const Args& a, hipStream_t stream) {
  const int64_t items = most_tiles(a);
  if (a.kv_dtype == TOPKV_FP8_E4M3) {
    if (a.dtype == TOPKV_BF16) launch<TOPKV_BF16, true>(a, items, stream);
    else launch<TOPKV_FP16, true>(a, items, stream);
  } else if (a.dtype == TOPKV_BF16) {
    launch<TOPKV_BF16, false>(a, items, stream);
  } else {
    launch<TOPKV_FP16, false>(a, items, stream);
  }
  return hipGetLastError() == hipSuccess ? TOPKV_OK : TOPKV_ERR_LAUNCH;
}

}  // namespace topkv_attend
