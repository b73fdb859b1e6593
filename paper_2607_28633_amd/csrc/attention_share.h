// attention_share.h - decode's division of a batch into equal shares, and the
// join of requests that were cut (attention_decode.hip, attention_latent.hip).
#ifndef TOPKV_ATTENTION_SHARE_H_
#define TOPKV_ATTENTION_SHARE_H_

#include "attention_mfma.h"

namespace topkv_attend {
namespace {

constexpr int kTile = 32;                // keys of a tile
constexpr int kLeast = 8;                // tiles of a share, at least: smaller pieces cost more to join than they save
constexpr int kSingle = 512;             // longest visible length that is never cut (one launch, no join)

struct Plan {
  int32_t shares;      // wanted; 0: one per request, whatever its length
  int32_t part_dim;    // value_dim, up to a multiple of 8
  float* part;         // [2 * share + 1 for a request's first piece][query head][part_dim]
  float2v* part_ml;    // the same without part_dim: maximum and sum
  bool by_request;     // what `cut` is indexed by: requests, or shares where these are fewer
  int4* cut;           // the request in pieces (of that number, or that starts in that share), its first share, how many (0: none)
};

struct Share {
  int32_t request;     // of the first tile; -1: the share is empty
  int32_t base;        // number of that request's first tile
  int32_t size;        // tiles of a share
  int32_t total;       // tiles of the batch
};

// Every request has at least one tile, so that those of no tokens are written too.
__device__ __forceinline__ int32_t tiles_of(const Args& a, int32_t r) {
  const int32_t p = clamped_len(a, r) - 1, n = key_span(a, p, p).count;
  return n < 1 ? 1 : (n + kTile - 1) / kTile;
}

template <int kWaves>
__device__ Share find_share(const Args& a, int32_t shares, int32_t share) {
  __shared__ Share s_got;
  if (threadIdx.x == 0) s_got.request = -1;
  const auto tiles = [&](int32_t r) { return tiles_of(a, r); };
  Scan<int32_t> n = scan_requests<int32_t, kWaves>(a.num_reqs, tiles);
  int32_t size = (n.total + shares - 1) / shares;
  size = size < kLeast ? kLeast : size;
  const int32_t first = share * size;
  if (n.holds(first)) {
    s_got.request = n.find(first, tiles);
    s_got.base = n.base;
  }
  __syncthreads();
  Share got = s_got;
  got.size = size;
  got.total = n.total;
  return got;
}

// Requests in pieces: a wave per (request or share, query head, 128 elements),
// 16 lanes with 8 elements each for every fourth piece, so that a wave reads
// whole lines and few of its loads wait for each other; with kDeep, for few
// requests of many pieces, a workgroup of four waves (1048576 tokens, one KV
// head, 512 pieces: 107 us with one wave, 96 with four; 64 requests of an
// e4m3 cache: 155 with one, 157 with four).
constexpr int kJoinWaves = 4;

template <int T, bool kDeep>
__global__ __launch_bounds__(64 * kJoinWaves) void kv_attention_join_kernel(Args a, Plan plan) {
  typedef typename Elem<T>::type elem;
  __shared__ float s_sum[kJoinWaves][16][9];
  const int32_t each = kDeep ? 1 : kJoinWaves, sets = (a.num_heads + each - 1) / each, entry = blockIdx.x / sets;
  const int4 cut = plan.cut[entry];
  const int32_t r = cut.x, share = cut.y, pieces = cut.z;
  const int wave = threadIdx.x >> 6;
  const int32_t head = (blockIdx.x - entry * sets) * each + (kDeep ? 0 : wave);
  if (pieces == 0 || head >= a.num_heads) return;
  const int lane = threadIdx.x & 63;
  const int64_t step = a.num_heads, at = 2 * (int64_t)share * step + head;   // piece k: slot 2 (first + k), the first one's next to it
  float top = -INFINITY;
  for (int32_t k = lane; k < pieces; k += 64) top = fmaxf(top, plan.part_ml[at + (k ? 2 * k : 1) * step][0]);
#pragma unroll
  for (int i = 32; i; i >>= 1) top = fmaxf(top, __shfl_xor(top, i, 64));
  const float base = top == -INFINITY ? 0.f : top;
  const int32_t d = blockIdx.y * 128 + (lane & 15) * 8;
  float sum = 0.f;
  float4v lo = {0.f, 0.f, 0.f, 0.f}, hi = lo;
  if (d < plan.part_dim) {
#pragma unroll 4
    for (int32_t k = (kDeep ? wave * 4 : 0) + (lane >> 4); k < pieces; k += kDeep ? 4 * kJoinWaves : 4) {
      const int64_t slot = at + (k ? 2 * k : 1) * step;
      const float2v ml = plan.part_ml[slot];
      const float4v* from = reinterpret_cast<const float4v*>(plan.part + slot * plan.part_dim + d);
      const float f = __builtin_amdgcn_exp2f(ml[0] - base);
      sum = fmaf(f, ml[1], sum);
      lo += from[0] * f;
      hi += from[1] * f;
    }
  }
  sum = sum_quarters(sum);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    lo[i] = sum_quarters(lo[i]);
    hi[i] = sum_quarters(hi[i]);
  }
  if constexpr (kDeep) {
    if (lane < 16) {
      s_sum[wave][lane][8] = sum;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s_sum[wave][lane][i] = lo[i];
        s_sum[wave][lane][i + 4] = hi[i];
      }
    }
    __syncthreads();
    if (wave > 0) return;
    sum = 0.f;
    lo = hi = float4v{0.f, 0.f, 0.f, 0.f};
    for (int w = 0; w < kJoinWaves; ++w) {
      sum += s_sum[w][lane & 15][8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        lo[i] += s_sum[w][lane & 15][i];
        hi[i] += s_sum[w][lane & 15][i + 4];
      }
    }
  }
  if (lane < 16 && d < a.value_dim) {
    elem* out = static_cast<elem*>(a.out) + (int64_t)r * a.out_stride + (int64_t)head * a.value_dim + d;
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
    if (a.out_wide && a.value_dim % 8 == 0) {
      *reinterpret_cast<uint4v*>(out) = u.w;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (d + i < a.value_dim) out[i] = u.e[i];
    }
  }
  if (a.lse && lane == 0 && blockIdx.y == 0)
    a.lse[(int64_t)r * a.num_heads + head] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

int64_t up16(int64_t x) { return (x + 15) / 16 * 16; }

// Shares that a call wants, 0 where no request can be long enough to be cut.
int32_t shares_for(const Args& a, int32_t resident, int32_t units) {
  const int64_t seen = (int64_t)a.bt_stride * a.page_size;
  const int64_t most = a.window > 0 && (int64_t)a.window + a.sinks < seen ? (int64_t)a.window + a.sinks : seen;
  if (most <= kSingle) return 0;
  const int32_t n = resident / units;
  return n < 1 ? 1 : n;
}

int64_t plan_bytes(const Args& a, int32_t shares) {
  if (shares == 0) return 0;
  const int64_t rows = 2 * (int64_t)shares * a.num_heads;
  return up16(rows * ((a.value_dim + 7) / 8 * 8) * 4) + up16(rows * 8) + (int64_t)shares * 16;
}

Plan make_plan(const Args& a, int32_t shares, void* workspace) {
  Plan p = {};
  p.shares = shares;
  if (shares > 0) {
    const int64_t rows = 2 * (int64_t)shares * a.num_heads;
    char* at = static_cast<char*>(workspace);
    p.part_dim = (a.value_dim + 7) / 8 * 8;
    p.part = reinterpret_cast<float*>(at);
    at += up16(rows * p.part_dim * 4);
    p.part_ml = reinterpret_cast<float2v*>(at);
    at += up16(rows * 8);
    p.cut = reinterpret_cast<int4*>(at);
    p.by_request = a.num_reqs <= shares;
  }
  return p;
}

void launch_join(const Args& a, const Plan& p, hipStream_t stream) {
  if (p.shares == 0) return;
  const bool deep = p.shares >= 16 * (int64_t)a.num_reqs;
  const int32_t sets = deep ? a.num_heads : (a.num_heads + kJoinWaves - 1) / kJoinWaves;
  const dim3 grid((unsigned)((p.by_request ? a.num_reqs : p.shares) * sets), (unsigned)((a.value_dim + 127) / 128));
  const dim3 block(64 * kJoinWaves);
  if (a.dtype == TOPKV_BF16) {
    if (deep) hipLaunchKernelGGL(HIP_KERNEL_NAME(kv_attention_join_kernel<TOPKV_BF16, true>), grid, block, 0, stream, a, p);
    else hipLaunchKernelGGL(HIP_KERNEL_NAME(kv_attention_join_kernel<TOPKV_BF16, false>), grid, block, 0, stream, a, p);
  } else {
    if (deep) hipLaunchKernelGGL(HIP_KERNEL_NAME(kv_attention_join_kernel<TOPKV_FP16, true>), grid, block, 0, stream, a, p);
    else hipLaunchKernelGGL(HIP_KERNEL_NAME(kv_attention_join_kernel<TOPKV_FP16, false>), grid, block, 0, stream, a, p);
  }
}

// Whether the grid stays a launch's (whatever num_reqs: a workspace for many requests serves fewer too).
bool launchable(const Args& a, int32_t shares, int32_t units) {
  const int64_t items = (shares > TOPKV_MAX_BATCH_REQS ? shares : TOPKV_MAX_BATCH_REQS) + 8;
  return items * units <= kMostGroups && (int64_t)shares * a.num_heads <= kMostGroups;
}

// Rows on addresses that the wide loads take.
bool rows_aligned(const Args& a) {
  const int64_t unit = a.kv_dtype == TOPKV_FP8_E4M3 ? 8 : 16;
  return a.head_dim % 8 == 0 && a.slot_bytes % unit == 0 && a.head_bytes % unit == 0 && a.page_bytes % unit == 0 &&
         a.value_bytes % unit == 0;
}

}  // namespace
}  // namespace topkv_attend

#endif  // TOPKV_ATTENTION_SHARE_H_
