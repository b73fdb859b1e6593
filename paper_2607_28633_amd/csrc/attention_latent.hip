// attention_latent.hip - one new token per request over a latent cache
// (planes = 1, rows of up to 576 elements whose front is also the value) on
// the matrix units.
//
// All query heads share one latent row, so a workgroup takes up to 64 of them
// and the row is read from memory once for all: 2 * 64 * (576 + 512) flops
// for 1152 bytes, still less than the matrix units do in the time the bytes
// take.  The output, 64 rows of 512, is too much for one wave: the eight waves
// of a workgroup share a tile of 32 keys.  For the scores a wave takes 16 keys,
// 16 rows and, where there are few rows, a half or a quarter of the elements;
// the parts meet in LDS, from where the weights come that a wave multiplies with
// its 64 elements of the values.  Three tiles are in LDS, straight from memory:
// one in use, and two asked for ahead, since a CU holds one workgroup.  Of
// these two only the later is under way while a tile is multiplied: the compiler,
// which does not see loads to LDS, waits for all loads where it uses the table
// entry that it asked for before them, once a tile.
#include <type_traits>

#include "attention_internal.h"
#include "attention_share.h"

namespace topkv_attend {

namespace {

constexpr int kWaves = 8;
constexpr int kThreads = 64 * kWaves;
constexpr int KD = 576, VD = 512;        // elements of a row and of its value, padded
constexpr int NC = KD / 8;               // 16-byte chunks of a row in LDS
constexpr int kTileBytes = kTile * KD * 2;
constexpr int kPieces = kTileBytes / 1024;               // wave-wide loads of a tile
constexpr int kLoads = (kPieces + kWaves - 1) / kWaves;  // of a wave
constexpr int kBuffers = 3;
constexpr int kResident = 256;           // workgroups that 256 CUs hold at once
constexpr float kSlack = 8.f;            // see attention_prompt.hip

template <int T, bool kF8, int RB, bool kCut>
__global__ __launch_bounds__(kThreads, 2) void kv_attention_latent_kernel(Args a, Plan plan) {
  typedef typename Elem<T>::vec8 vec8;
  typedef typename Elem<T>::type elem;
  constexpr int kRows = 16 * RB;
  __shared__ __attribute__((aligned(16))) char s_tile[kBuffers][kTileBytes];
  constexpr int kParts = 4 / RB;                                 // of the elements, in the first product
  constexpr int kSteps = (KD / 32 + kParts - 1) / kParts;        // of 32 elements, in a part
  constexpr int kPitch = kTile + 4;                              // floats of a row of scores: rows start 4 banks apart
  constexpr bool kEach = RB < 4;                                 // every wave makes all weights, or each wave its own for all
  __shared__ __attribute__((aligned(16))) float s_score[kEach ? kParts : 1][kEach ? kRows : 1][kPitch];
  __shared__ __attribute__((aligned(16))) elem s_weight[kEach ? 1 : kRows][kTile];
  __shared__ float s_top[2][kEach ? 1 : kRows], s_sum[2][kEach ? 1 : kRows];

  const int wave = threadIdx.x >> 6;
  const int key_half = wave & 1, row_block = (wave >> 1) % RB, part = (wave >> 1) / RB;   // of the wave's scores
  const int32_t groups = (a.group + kRows - 1) / kRows;
  const int32_t units = a.kv_heads * groups, eight = blockIdx.x / (8 * units), within = blockIdx.x - eight * 8 * units;
  const int32_t share = eight * 8 + (within & 7), sub = within >> 3;   // over the XCDs as in attention_decode.hip
  const int32_t kv_head = sub % a.kv_heads, first_row = sub / a.kv_heads * kRows;
  const char* cache = a.cache + (int64_t)kv_head * a.head_bytes;
  const int32_t chunks = a.head_dim / 8;
  constexpr int kChunkBytes = kF8 ? 8 : 16;

  Share sh = {share, 0, 0, 0};
  int32_t tile_at = 0, tile_end = 1;
  if constexpr (kCut) {
    if (share >= plan.shares) return;
    sh = find_share<kWaves>(a, plan.shares, share);
    if (!plan.by_request && sub == 0 && threadIdx.x == 0) plan.cut[share] = make_int4(0, 0, 0, 0);
    if (sh.request < 0) return;
    tile_at = share * sh.size;
    tile_end = tile_at + sh.size < sh.total ? tile_at + sh.size : sh.total;
  } else {
    if (share >= a.num_reqs) return;
  }
  if (chunks < NC) {                                             // padding stays zero: loads leave it alone
    for (int i = threadIdx.x; i < kBuffers * kTileBytes / 16; i += kThreads)
      *reinterpret_cast<uint4v*>(&s_tile[0][0] + i * 16) = uint4v{0, 0, 0, 0};
    __syncthreads();
  }

  for (int32_t request = sh.request; tile_at < tile_end; ++request) {
  int lane = threadIdx.x & 63;
  asm volatile("" : "+v"(lane));                                 // addresses made from it stay in the loop: registers
  const int row = lane & 15, quad = lane >> 4;
  const int32_t pos = clamped_len(a, request) - 1;
  const Span span = key_span(a, pos, pos);
  int32_t begin = 0, end = span.count;
  bool whole = true, opens = false;
  if constexpr (kCut) {
    const int32_t tiles = span.count < 1 ? 1 : (span.count + kTile - 1) / kTile, from = tile_at - sh.base;
    const int32_t to = tile_end - sh.base < tiles ? tile_end - sh.base : tiles;
    opens = from == 0;
    whole = opens && to == tiles;
    begin = from * kTile;
    end = to * kTile < span.count ? to * kTile : span.count;
    if (opens && (!whole || plan.by_request) && sub == 0 && threadIdx.x == 0)
      plan.cut[plan.by_request ? request : share] =
          make_int4(request, share, whole ? 0 : (sh.base + tiles - 1) / sh.size - share + 1, 0);
    tile_at = sh.base + to;
    sh.base += tiles;
  } else {
    tile_at = tile_end;
  }

  const int32_t* table = a.tables + (int64_t)request * a.bt_stride;
  const auto ask = [&](int32_t first) -> int32_t {
    const int32_t v = first + (lane & 31);
    return v < end ? table[page_of(a, (uint32_t)key_position(span, v))] : -1;
  };
  const auto locate = [&](int32_t first, int32_t entry) -> int64_t {
    const int32_t v = first + (lane & 31);
    if (v >= end || entry < 0 || entry >= a.num_pages) return -1;
    const uint32_t j = (uint32_t)key_position(span, v);
    return (int64_t)entry * a.page_bytes + (int64_t)(j - page_of(a, j) * (uint32_t)a.page_size) * a.slot_bytes;
  };
  // load i of the wave: 64 places of 16 bytes of the tile
  uint2v raw[kF8 ? kLoads : 1];
  const auto fetch = [&](int buf, int64_t off) {
    const int lo = off < 0 ? 0 : (int)(uint32_t)off, hi = off < 0 ? 0 : (int)(off >> 32);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int piece = i * kWaves + wave;
      if (piece < kPieces) {
        const int place = piece * 64 + lane, r = place / NC, c = (place - r * NC) ^ swizzle<NC>(r);
        const char* from =
            cache + (int64_t)((uint64_t)(uint32_t)__shfl(hi, r, 64) << 32 | (uint32_t)__shfl(lo, r, 64)) + c * kChunkBytes;
        if (c < chunks) {
          if constexpr (kF8) raw[i] = *reinterpret_cast<const uint2v*>(from);
          else if constexpr (kCut) load_once_to_lds(s_tile[buf] + piece * 1024, from);
          else load_to_lds(s_tile[buf] + piece * 1024, from);
        }
      }
    }
  };
  // rows without a key as zeros, whatever their place holds; an 8-bit cache is widened on the way
  const auto settle = [&](int buf, uint32_t there) {
    if (!kF8 && there == ~0u) return;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int piece = i * kWaves + wave;
      if (piece < kPieces) {
        const int place = piece * 64 + lane, r = place / NC, c = (place - r * NC) ^ swizzle<NC>(r);
        const bool is = there >> r & 1;
        uint4v* to = reinterpret_cast<uint4v*>(s_tile[buf] + place * 16);
        if (c < chunks) {
          if constexpr (kF8) *to = is ? widen<T>(raw[i]) : uint4v{0, 0, 0, 0};
          else if (!is) *to = uint4v{0, 0, 0, 0};
        }
      }
    }
  };

  // tiles i, i + 1, i + 2: which keys are there
  int32_t entry = ask(begin);
  int64_t off = locate(begin, entry);
  entry = ask(begin + kTile);
  uint32_t there = (uint32_t)__ballot(off >= 0), there1 = 0, there2 = 0;
  if (begin < end) fetch(0, off);
  if constexpr (kF8) {
    if (begin < end) settle(0, there);
  }
  off = locate(begin + kTile, entry);
  entry = ask(begin + 2 * kTile);
  there1 = (uint32_t)__ballot(off >= 0);
  if (begin + kTile < end) fetch(1, off);

  vec8 q[kSteps];
  {
    const int32_t h = first_row + row_block * 16 + row;
    const char* from =
        static_cast<const char*>(a.q) + ((int64_t)request * a.q_stride + (int64_t)(kv_head * a.group + h) * a.head_dim) * 2;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int d = (s * kParts + part) * 32 + quad * 8;
      union {
        uint4v w;
        vec8 v;
      } u;
      u.w = uint4v{0, 0, 0, 0};
      if (h < a.group && d < a.head_dim) u.w = *reinterpret_cast<const uint4v*>(from + 2 * d);
      q[s] = u.v;
    }
  }
  float4v acc[RB][4];
  float m[RB], l[RB];
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    m[b] = -INFINITY;
    l[b] = 0.f;
#pragma unroll
    for (int t = 0; t < 4; ++t) acc[b][t] = float4v{0.f, 0.f, 0.f, 0.f};
  }

  int buf = 0;
  for (int32_t first = begin; first < end; first += kTile) {
    const int next = buf + 1 < kBuffers ? buf + 1 : 0, last = next + 1 < kBuffers ? next + 1 : 0;
    if constexpr (!kF8) {
      // this wave's part of the tile has landed when no more than the next tile's loads (4 at least) are under way; those
      // are waited for below, where the compiler uses `entry`
      // (narrower rows: some of a tile's loads may have no lane to them and are never issued)
      if (first + kTile < end && chunks == NC) asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
      else wait_loads();
      settle(buf, there);
    }
    __syncthreads();                                             // the tile is whole; the one before it and its scores are done with
    if constexpr (kF8) {
      if (first + kTile < end) settle(next, there1);
    }
    off = locate(first + 2 * kTile, entry);
    there2 = (uint32_t)__ballot(off >= 0);
    if (first + 2 * kTile < end) {
      entry = ask(first + 3 * kTile);
      fetch(last, off);
    }
    const char* tile = s_tile[buf];
    int here = lane;
    asm volatile("" : "+v"(here));                               // and these in the tile's loop
    const int row = here & 15, quad = here >> 4;
    float4v x = {0.f, 0.f, 0.f, 0.f};
    {
      const int r = key_half * 16 + row;
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        const int n = s * kParts + part;
        if (kSteps * kParts > KD / 32 && n >= KD / 32) break;    // the last part is a step short
        const vec8 k = *reinterpret_cast<const vec8*>(tile + (r * NC + ((n * 4 + quad) ^ swizzle<NC>(r))) * 16);
        x = Elem<T>::mfma16(k, q[s], x);
      }
    }
    vec8 p[RB];
    if constexpr (kEach) {
    *reinterpret_cast<float4v*>(&s_score[part][row_block * 16 + row][key_half * 16 + quad * 4]) = x;
    __syncthreads();
    // lane (row, quad) takes keys 8 quad .. + 7 of its row: the layout the second product wants
#pragma unroll
    for (int b = 0; b < RB; ++b) {
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; e += 4) {
        float4v sum = *reinterpret_cast<const float4v*>(&s_score[0][b * 16 + row][quad * 8 + e]);
#pragma unroll
        for (int n = 1; n < kParts; ++n) sum += *reinterpret_cast<const float4v*>(&s_score[n][b * 16 + row][quad * 8 + e]);
#pragma unroll
        for (int i = 0; i < 4; ++i) y[e + i] = sum[i];
      }
      if (there != ~0u) {
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = there >> (quad * 8 + i) & 1 ? y[i] : -INFINITY;
      }
      float top = y[0];
#pragma unroll
      for (int i = 1; i < 8; ++i) top = fmaxf(top, y[i]);
      top = reference<T>(max_quarters(top), a.scale, kSlack);
      if (__any(top - m[b] > kSlack)) {
        const float up = fmaxf(m[b], top), fall = m[b] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[b] - up);
        m[b] = up;
        l[b] *= fall;
#pragma unroll
        for (int t = 0; t < 4; ++t) acc[b][t] *= fall;
      }
      const float base = m[b] == -INFINITY ? 0.f : m[b];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float w = weight_of(y[i], a.scale, base);
        l[b] += w;
        p[b][i] = (elem)w;                                       // rounded for the matrix units, its sum is not
      }
    }
    } else {
    // 64 rows: making all weights eight times over costs more than two exchanges (64 heads 109 us, 94 so; 16 heads 59, 64 so)
    if (there != ~0u) {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = there >> (key_half * 16 + quad * 4 + i) & 1 ? x[i] : -INFINITY;
    }
    const float best = reference<T>(max_quarters(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]))), a.scale, kSlack);
    if (quad == 0) s_top[key_half][row_block * 16 + row] = best;
    __syncthreads();
    float fall_mine = 1.f, base_mine = 0.f;
#pragma unroll
    for (int b = 0; b < RB; ++b) {                               // every wave keeps every row's maximum
      const float top = fmaxf(s_top[0][b * 16 + row], s_top[1][b * 16 + row]);
      float fall = 1.f;
      if (__any(top - m[b] > kSlack)) {
        const float up = fmaxf(m[b], top);
        fall = m[b] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[b] - up);
        m[b] = up;
#pragma unroll
        for (int t = 0; t < 4; ++t) acc[b][t] *= fall;
      }
      if (b == row_block) {
        fall_mine = fall;
        base_mine = m[b] == -INFINITY ? 0.f : m[b];
      }
    }
    l[0] *= fall_mine;                                           // of the wave's own rows and keys
    union {
      elem e[4];
      uint2v w;
    } u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float w = weight_of(x[i], a.scale, base_mine);
      l[0] += w;
      u.e[i] = (elem)w;
    }
    *reinterpret_cast<uint2v*>(&s_weight[row_block * 16 + row][key_half * 16 + quad * 4]) = u.w;
    __syncthreads();
#pragma unroll
    for (int b = 0; b < RB; ++b) p[b] = *reinterpret_cast<const vec8*>(&s_weight[b * 16 + row][quad * 8]);
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) {                                // 16 elements of the value at a time, by columns
      union {
        uint2v h[2];
        vec8 v;
      } u;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = quad * 8 + e * 4 + (row >> 2), c = wave * 8 + t * 2 + (row >> 1 & 1);
        u.h[e] = read_transposed(tile + (r * NC + (c ^ swizzle<NC>(r))) * 16 + (row & 1) * 8);
      }
#pragma unroll
      for (int b = 0; b < RB; ++b) acc[b][t] = Elem<T>::mfma16(u.v, p[b], acc[b][t]);
    }
    there = there1;
    there1 = there2;
    buf = next;
  }

  if constexpr (!kEach) {
    const float sum = sum_quarters(l[0]);
    if (quad == 0) s_sum[key_half][row_block * 16 + row] = sum;
    __syncthreads();
  }
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    const int32_t h = first_row + b * 16 + row, head = kv_head * a.group + h;
    float sum;
    if constexpr (kEach) sum = sum_quarters(l[b]);
    else sum = s_sum[0][b * 16 + row] + s_sum[1][b * 16 + row];
    if (h >= a.group) continue;
    const int64_t slot = (2 * (int64_t)share + opens) * a.num_heads + head;
    const float inv = sum == 0.f ? 0.f : a.v_scale / sum;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int d = wave * 64 + t * 16 + quad * 4;
      if (!whole) {
        if (d < plan.part_dim) *reinterpret_cast<float4v*>(plan.part + slot * plan.part_dim + d) = acc[b][t];
        continue;
      }
      elem* out = static_cast<elem*>(a.out) + (int64_t)request * a.out_stride + (int64_t)head * a.value_dim + d;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (d + e < a.value_dim) out[e] = (elem)(sum == 0.f ? 0.f : acc[b][t][e] * inv);
    }
    if (wave == 0 && quad == 0) {
      if (!whole) plan.part_ml[slot] = float2v{m[b], sum};
      else if (a.lse)
        a.lse[(int64_t)request * a.num_heads + head] = sum == 0.f ? -INFINITY : (m[b] + __builtin_amdgcn_logf(sum)) * kLn2;
    }
  }
  __syncthreads();                                               // tiles and scores are free again
  }
}

// Row blocks of 16 that a workgroup takes.
int row_blocks(const Args& a) { return a.group <= 16 ? 1 : a.group <= 32 ? 2 : 4; }

int32_t units(const Args& a) {
  const int32_t rows = 16 * row_blocks(a);
  return a.kv_heads * ((a.group + rows - 1) / rows);
}

int32_t wanted_shares(const Args& a) { return shares_for(a, kResident, units(a)); }

template <int T, bool kF8>
void launch(const Args& a, const Plan& p, hipStream_t stream) {
  const int64_t items = p.shares > 0 ? p.shares : a.num_reqs;
  const dim3 grid((unsigned)((items + 7) / 8 * 8 * units(a))), block(kThreads);
#define TOPKV_LATENT(RB)                                                                                                  \
  do {                                                                                                                    \
    if (p.shares > 0)                                                                                                     \
      hipLaunchKernelGGL(HIP_KERNEL_NAME(kv_attention_latent_kernel<T, kF8, RB, true>), grid, block, 0, stream, a, p);    \
    else                                                                                                                  \
      hipLaunchKernelGGL(HIP_KERNEL_NAME(kv_attention_latent_kernel<T, kF8, RB, false>), grid, block, 0, stream, a, p);   \
  } while (0)
  if (row_blocks(a) == 1) TOPKV_LATENT(1);
  else if (row_blocks(a) == 2) TOPKV_LATENT(2);
  else TOPKV_LATENT(4);
#undef TOPKV_LATENT
  launch_join(a, p, stream);
}

}  // namespace

bool latent_takes(const Args& a) {
  return rows_aligned(a) && a.value_bytes == 0 && a.head_dim > 128 && a.head_dim <= KD && a.value_dim <= VD &&
         launchable(a, wanted_shares(a), units(a));
}

int64_t latent_workspace(const Args& a) { return plan_bytes(a, wanted_shares(a)); }

topkv_status_t run_latent(const Args& a, void* workspace, hipStream_t stream) {
  const Plan p = make_plan(a, wanted_shares(a), workspace);
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
